// Arguments of the cross-attention kernels after host validation (strides in
// elements), and how a call is divided.
#pragma once

#include <hip/hip_runtime.h>
#include <stddef.h>
#include <stdint.h>

#include "cache_args.h"

namespace sva {

struct CrossArgs {
  HeadsView q, k, v, out;        // forward: out is written; backward: read
  HeadsView dout, dq, dk, dv;    // backward
  const int32_t* lens;           // [B] keys of an entry, null: M
  const uint8_t* mask;           // [B, M], null: none
  int64_t mask_b;
  uint32_t* bits;                // with a mask: [B, ceil(M / 32)], bit j of word i: key 32i + j is seen
  int32_t* seen;                 // with a mask: [B], keys up to the last seen one
  float* lse;                    // [B, H, N]; forward: written where not null; backward: read
  float* part;                   // partial results where keys (backward: or rows) are divided
  float* part_kv;                // backward: partial dK and dV
  float2* stat;                  // forward: (m, l) of a partial row; backward: (lse in log2 units, delta) of a row
  float* stat_l;                 // forward: a partial row's sum of unrounded weights
  int B, H, Hkv, G, N, M, R;     // G = H / Hkv heads share keys; R = G * N rows of a kv head
  float scale, scale_log2;
  int D;
  int tiles, splits;             // row tiles of a kv head; parts its keys are divided into
  int run;                       // row tiles that a workgroup takes one after the other (one where keys are divided)
  int key_tiles, row_splits;     // backward: 128-key tiles, parts the rows are divided into
  int wgs, kv_wgs;               // workgroups of the launches
};

// How a call is divided, and its workspace: offsets of what CrossArgs points to.
struct CrossShape {
  int few;                       // 16 rows at most: the waves divide the keys
  int narrow;                    // 16 rows a wave (64 a workgroup), else 32 (128)
  int run, tiles, splits, key_tiles, row_splits;
  size_t bits_at, seen_at, stat_at, stat_l_at, part_at, part_kv_at, ws_bytes;
};
CrossShape cross_shape(int B, int Hkv, int G, int N, int M, int D, bool mask, bool grad);
CrossShape cross_grad_shape(int B, int Hkv, int G, int N, int M, int D, bool mask);

hipError_t launch_cross_bits(const CrossArgs& a, hipStream_t stream);
hipError_t launch_cross_attention(const CrossArgs& a, const CrossShape& s, hipStream_t stream);
hipError_t launch_cross_attention_grad(const CrossArgs& a, const CrossShape& s, hipStream_t stream);

}  // namespace sva
