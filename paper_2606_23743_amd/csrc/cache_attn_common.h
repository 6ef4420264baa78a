// What the kernels of the attention over a paged cache share (cache_attn_kernel.h,
// cache_attn_tile.h, cache_attention.hip).
#pragma once

#include "attn_w16.h"
#include "cache_attn_plan.h"

namespace sva {
namespace cattn {

using attn::bf16x2;
using attn::bf16x8;
using attn::f32x2;
using attn::f32x4;
using attn::u32x2;
using attn::u32x4;

// four codes (bytes) -> four bf16 values in two dwords
template <int FMT>
__device__ __forceinline__ u32x2 widen4(uint32_t c) {
  u32x2 o;
  if constexpr (FMT == kCacheE4m3) {
    o[0] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(c, 1.0f, false));
    o[1] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(c, 1.0f, true));
  } else {
    // whole numbers up to 127 in float32: the upper halves are their bf16 values
    const float a = (float)((int)(c << 24) >> 24), b = (float)((int)(c << 16) >> 24);
    const float d = (float)((int)(c << 8) >> 24), e = (float)((int)c >> 24);
    o[0] = __builtin_amdgcn_perm(__float_as_uint(b), __float_as_uint(a), 0x07060302u);
    o[1] = __builtin_amdgcn_perm(__float_as_uint(e), __float_as_uint(d), 0x07060302u);
  }
  return o;
}

// weights times V scales as NP B operands: rounded to bf16 (NP = 1, bf16 results), or as
// the sum of three bf16 values, which holds all 24 bits (float32 results: with two
// parts they were off by 1.4e-6 of their norm, with three by what the logits are).
// A bf16 result's own rounding is 1.7e-3 of its norm, and weights rounded as well make that
// 1.9e-3 to 2.4e-3, as in the whole-sequence attention; the results differ by up to 2.7e-3
// from those of float32 weights (float32 results by 7e-7 from float64).  What all 24 bits cost,
// us of bf16 / float32 results: 8 sequences of 32,768 keys, 6 heads and 128 rows 170 / 234 (int8),
// 179 / 247 (bf16); 2 of 223,200 e4m3 keys, 8 heads and 48 rows 199 / 244; 48 of 16,384, four
// rows, 268 / 268, where HBM bounds both.
template <int QT, int NP>
__device__ __forceinline__ void weight_operands(const float (&p)[QT][8], bf16x8 (&part)[NP][QT]) {
#pragma unroll
  for (int qt = 0; qt < QT; ++qt) {
    float a[8];
#pragma unroll
    for (int e = 0; e < 8; ++e) a[e] = p[qt][e];
#pragma unroll
    for (int n = 0; n < NP; ++n) {
      u32x4 h;
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        h[e] = __builtin_bit_cast(uint32_t, attn::cvt2(a[2 * e], a[2 * e + 1]));
        a[2 * e] -= __uint_as_float(h[e] << 16);
        a[2 * e + 1] -= __uint_as_float(h[e] & 0xFFFF0000u);
      }
      part[n][qt] = __builtin_bit_cast(bf16x8, h);
    }
  }
}

// values that every lane holds alike, as scalars
__device__ __forceinline__ int uniform(int x) { return __builtin_amdgcn_readfirstlane(x); }
__device__ __forceinline__ int64_t uniform(int64_t x) {
  const uint32_t lo = __builtin_amdgcn_readfirstlane((uint32_t)x), hi = __builtin_amdgcn_readfirstlane((uint32_t)(x >> 32));
  return (int64_t)((uint64_t)hi << 32 | lo);
}

// lane l's value
__device__ __forceinline__ int64_t lane_value(int64_t x, int l) {
  const uint32_t lo = __builtin_amdgcn_readlane((uint32_t)x, l), hi = __builtin_amdgcn_readlane((uint32_t)(x >> 32), l);
  return (int64_t)((uint64_t)hi << 32 | lo);
}
// sums over lanes 0 .. l, in each lane l (DPP: within rows of 16 lanes, then a row's last
// lane to the next row, then lane 31 to the upper half)
template <int CTRL, int ROWS>
__device__ __forceinline__ int64_t moved(int64_t x) {
  const uint32_t lo = __builtin_amdgcn_update_dpp(0, (int)(uint32_t)x, CTRL, ROWS, 0xf, false);
  const uint32_t hi = __builtin_amdgcn_update_dpp(0, (int)(x >> 32), CTRL, ROWS, 0xf, false);
  return (int64_t)((uint64_t)hi << 32 | lo);
}
__device__ __forceinline__ int64_t wave_scan(int64_t x) {
  x += moved<0x111, 0xf>(x);
  x += moved<0x112, 0xf>(x);
  x += moved<0x114, 0xf>(x);
  x += moved<0x118, 0xf>(x);
  x += moved<0x142, 0xa>(x);
  x += moved<0x143, 0xc>(x);
  return x;
}

// Places of all segments, and the entry that holds a place, by one wave.  Each lane sums
// B / 64 neighbouring entries, one scan over the lanes gives every lane's first place, and the
// lane that holds what is looked for is taken apart in the same way (up to 64 entries: one
// look at memory in all; 4,096: two).
struct Finder {
  const CacheAttnArgs& a;
  int rows, begin;
  int per;                       // entries of a lane
  int len0, cnt0;                // per = 1: the lane's entry
  int64_t incl;                  // places of this lane's entries and all before them
  int64_t total;

  __device__ __forceinline__ Entry of(int len, int cnt) const {
    return entry_of(len, cnt, a.max_pages << a.c.log2_page, a.T, a.G, rows, a.kn.p != nullptr, begin);
  }
  // b alike in all lanes
  __device__ __forceinline__ Entry at(int b) const { return of(uniform(len_at(b)), uniform(cnt_at(b))); }
  __device__ __forceinline__ int len_at(int b) const { return a.lens[min(b, a.B - 1)]; }
  __device__ __forceinline__ int cnt_at(int b) const { return a.counts ? a.counts[min(b, a.B - 1)] : a.T; }

  // units and segments of n entries from b on
  struct Sums {
    int64_t units, segments;
  };
  __device__ __forceinline__ Sums one(int len, int cnt) const {
    const Entry e = of(len, cnt);
    const int64_t s = (int64_t)e.tiles * a.c.heads;
    return {e.units * s, s};
  }
  __device__ __forceinline__ Sums sums(int b, int n) const {
    Sums x{0, 0};
    constexpr int UN = 8;                          // loads on their way together
    for (int j = 0; j < n; j += UN) {
      int len[UN], cnt[UN];
#pragma unroll
      for (int k = 0; k < UN; ++k) {
        len[k] = len_at(b + j + k);
        cnt[k] = cnt_at(b + j + k);
      }
#pragma unroll
      for (int k = 0; k < UN; ++k) {
        const Sums y = one(len[k], cnt[k]);
        x.units += j + k < n ? y.units : 0;
        x.segments += j + k < n ? y.segments : 0;
      }
    }
    return x;
  }
  __device__ __forceinline__ int64_t places(Sums s) const { return begin < 0 ? s.segments : s.units + begin * s.segments; }

  __device__ __forceinline__ Finder(const CacheAttnArgs& args, int rows_, int grid)
      : a(args), rows(rows_), begin(args.divide ? 0 : -1), per((args.B + 63) >> 6), len0(0), cnt0(0) {
    const int lane = threadIdx.x & 63, n = min(max(a.B - lane * per, 0), per);
    Sums s{0, 0};
    if (per == 1) {
      len0 = len_at(lane);
      cnt0 = cnt_at(lane);
      const Sums y = one(len0, cnt0);
      if (n > 0) s = y;
    } else {
      s = sums(lane * per, n);
    }
    incl = wave_scan(places(s));
    total = lane_value(incl, 63);
    if (a.divide && begin_of(total, grid) > 0) {
      begin = begin_of(total, grid);
      incl += begin * wave_scan(s.segments);
      total = lane_value(incl, 63);
    }
  }

  // the entry that holds place x < total, or (want >= 0) entry want; which it is and its first place
  __device__ __forceinline__ Entry locate(int64_t x, int want, int& b, int64_t& first) const {
    const int lane = threadIdx.x & 63;
    int64_t in = incl;
    int lo = 0, each = per, len = len0, cnt = cnt0;
    first = 0;
    for (;;) {
      const int k = want >= 0 ? (want - lo) / each : __builtin_ctzll(__builtin_amdgcn_ballot_w64(first + in > x));
      if (k > 0) first += lane_value(in, k - 1);
      lo += k * each;
      if (each == 1) {
        b = lo;
        return of(__builtin_amdgcn_readlane(len, k), __builtin_amdgcn_readlane(cnt, k));
      }
      const int n = min(each, a.B - lo);
      each = (n + 63) >> 6;
      const int m = min(max(n - lane * each, 0), each);
      if (each == 1) {
        len = len_at(lo + lane);
        cnt = cnt_at(lo + lane);
        in = wave_scan(m > 0 ? places(one(len, cnt)) : 0);
      } else {
        in = wave_scan(places(sums(lo + lane * each, m)));
      }
    }
  }
};

// A partial result in the workspace: for each 16-row tile, 4 x 64 x JT floats in the
// order of the join's lanes (channels JT * (4g + w) .. + JT - 1 of row i at [w][16g + i]),
// then every row's reference, then every row's sum.
template <int D>
struct Part {
  static constexpr int JT = D > 64 ? 8 : 4;
  static constexpr int kTile = kWaves * 64 * JT;
  static __host__ __device__ constexpr int floats(int tiles) { return tiles * (kTile + 32); }
  static __device__ __forceinline__ int at(int tile, int w, int lane) { return tile * kTile + (w * 64 + lane) * JT; }
  static __device__ __forceinline__ int ref(int tiles, int row) { return tiles * kTile + row; }
  static __device__ __forceinline__ int sum(int tiles, int row) { return tiles * (kTile + 16) + row; }
};

template <int D>
__device__ __forceinline__ void store_row(const CacheAttnArgs& a, int b, int h, int t, int d0,
                                          const float* y) {
  constexpr int JT = D > 64 ? 8 : 4;
  const int64_t at = b * a.out.sb + h * a.out.sh + t * a.out.sn + d0;
  if (a.out_f32) {
    float* o = static_cast<float*>(a.out.p) + at;
#pragma unroll
    for (int e = 0; e < JT; e += 4) *reinterpret_cast<float4*>(o + e) = make_float4(y[e], y[e + 1], y[e + 2], y[e + 3]);
  } else {
    uint16_t* o = static_cast<uint16_t*>(a.out.p) + at;
    uint32_t w[JT / 2];
#pragma unroll
    for (int e = 0; e < JT / 2; ++e) w[e] = __builtin_bit_cast(uint32_t, attn::cvt2(y[2 * e], y[2 * e + 1]));
    if constexpr (JT == 8) *reinterpret_cast<uint4*>(o) = make_uint4(w[0], w[1], w[2], w[3]);
    else *reinterpret_cast<uint2*>(o) = make_uint2(w[0], w[1]);
  }
}

constexpr float kLn2 = 0.69314718055994530942f;

}  // namespace cattn
}  // namespace sva
