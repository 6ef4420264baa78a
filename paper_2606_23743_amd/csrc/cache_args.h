// Arguments of the rotary, cache and cache-attention kernels after host
// validation (strides in elements).
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

namespace sva {

// A dimension of a launch holds fewer than 2^32 threads.  go(first, n) launches workgroups
// first .. first + n - 1 of `groups`: all of them but for tensors of hundreds of millions of tokens.
template <class Go>
void launch_slices(int64_t groups, int threads, Go go) {
  const int64_t most = UINT32_MAX / threads;
  for (int64_t first = 0; first < groups; first += most) {
    const int64_t left = groups - first;
    go((int)first, (unsigned)(left < most ? left : most));
  }
}

struct HeadsView {
  void* p;
  int64_t sb, sh, sn;
  int heads;
};

// rotary.hip
struct RotaryArgs {
  HeadsView qi, qo, ki, ko;      // ki.heads == 0: no K
  const double* freq;
  const int32_t* pos;
  int64_t pos_b;
  const int32_t* axis;           // several axes: of each pair; null: one, position n of an entry at pos[n]
  int64_t pos_n, pos_a;          // several axes: strides of tokens and axes
  int axes;
  bool pos_f32;                  // several axes: positions are float32
  int B, N, D, rot;
  float magnitude;
  bool f32, half, backward;
  int piece;                     // bytes of an access: 16, 8, 4 or (bf16) 2
  bool ragged;                   // piece 8 or 4: the turned part (each half) and the rest hold 16 bytes or are none
  bool copy;                     // channels from rot on have to be copied
};
hipError_t launch_rotary(const RotaryArgs& a, hipStream_t stream);

// cache_rw.hip
enum CacheFormat { kCacheBf16 = 0, kCacheE4m3 = 1, kCacheInt8 = 2 };

struct CacheView {
  void* k;
  void* v;
  float* ks;
  float* vs;
  int format, num_pages, heads, log2_page, D;
};
struct CacheRowsArgs {
  CacheView c;
  HeadsView k, v;
  const int32_t* slots;
  int64_t slots_b;
  int B, N;
  bool f32;
  int first;                     // a launch's first workgroup
};
hipError_t launch_cache_write(const CacheRowsArgs& a, hipStream_t stream);
hipError_t launch_cache_read(const CacheRowsArgs& a, hipStream_t stream);

// cache_attention.hip
struct CacheAttnArgs {
  CacheView c;
  HeadsView q, kn, vn, out;      // kn.p null: no drafted keys
  const int32_t* table;
  const int32_t* lens;
  const uint8_t* mask;           // null: causal
  int64_t mask_b;
  const int32_t* counts;
  float* ws;
  float* lse;
  int B, H, G, T, max_pages;     // G = H / kv heads
  float scale_log2;
  bool out_f32;
  bool divide;                   // whether a sequence's keys may be divided among workgroups
};
// How a call is run, and its workspace.
struct CacheAttnShape {
  bool shared;                   // waves share their keys (cache_attn_tile.h), or each has its own
  int tiles;                     // 16-row tiles of a workgroup: 1 to 3; shared: 4 or 8
  int wgs;                       // workgroups
  bool split;                    // whether a sequence's keys may be divided
  size_t ws_bytes;
};
CacheAttnShape cache_attn_shape(const CacheAttnArgs& a);
hipError_t launch_cache_attention(const CacheAttnArgs& a, hipStream_t stream);
// one cache format each
hipError_t launch_cache_attention_bf16(const CacheAttnArgs& a, const CacheAttnShape& s, hipStream_t stream);
hipError_t launch_cache_attention_e4m3(const CacheAttnArgs& a, const CacheAttnShape& s, hipStream_t stream);
hipError_t launch_cache_attention_int8(const CacheAttnArgs& a, const CacheAttnShape& s, hipStream_t stream);

}  // namespace sva
