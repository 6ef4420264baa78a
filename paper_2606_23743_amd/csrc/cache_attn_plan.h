// How the keys of a call are divided among workgroups (cache_attn_kernel.h,
// cache_attention.hip).  Host and device code, so that the division can be
// checked without a GPU.
//
// A segment is one (batch entry, cache head, row tile); its keys are cut into
// units of 128 (a 32-key step of each of four waves): first the cached keys,
// then the drafted ones, at least one unit.  The units of all segments, in the
// order (entry, head, tile, key), are dealt to n workgroups in runs of equal
// length: workgroup i takes units i*U/n .. (i+1)*U/n - 1 of U.  However ragged the
// lengths, every workgroup then reads the same number of keys; a run may cross
// segments, and a segment whose units went to several workgroups is joined from
// their partial results afterwards.  Short caches are not divided (their segments count as
// one unit each): joining would cost more than it gives.  A workgroup leaves at most two parts:
// slot 2i for a run that begins inside a segment, 2i + 1 for one that begins with a
// segment and ends inside it.
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

namespace sva {
namespace cattn {

constexpr int kUnit = 128;       // keys of a unit
// Segments of at most so many units are not divided: the join's launch takes longer than the
// units one after the other (us a call, divided / whole, 8 cache heads of 500 tokens: one
// sequence 18.4 / 15.8, 64 of them 27.4 / 20.9; 16 of 900 tokens 19.9 / 21.4, one of 1,900
// 17.6 / 30.6)
constexpr int kWholeUnits = 6;
constexpr int kWaves = 4;

// Workgroups per CU (waves per SIMD) of cache_attn_kernel with QT row tiles: at D = 64 and
// one tile a third finds its registers, and brings 943 MB from 102 us to 90; at D = 128 it
// would spill (137 us to 155 for 840 MB)
constexpr int wave_residents(int D, int QT) { return D == 64 && QT == 1 ? 3 : 2; }

struct Entry {                   // one batch entry
  int len;                       // cached tokens
  int cnt;                       // drafted tokens
  int cached_units, units;       // of each of its segments
  int tiles;                     // row tiles
  int span;                      // units of a segment in the division: 1 where segments are not divided
};

__host__ __device__ __forceinline__ Entry entry_of(int len, int cnt, int max_len, int T, int G, int rows, bool drafts,
                                                         bool divide) {
  Entry e;
  e.len = len < 0 ? 0 : (len > max_len ? max_len : len);
  e.cnt = cnt < 0 ? 0 : (cnt > T ? T : cnt);
  e.cached_units = (int)(((int64_t)e.len + kUnit - 1) / kUnit);
  e.units = e.cached_units + (drafts ? (e.cnt + kUnit - 1) / kUnit : 0);
  if (e.units < 1) e.units = 1;
  e.tiles = (int)(((int64_t)e.cnt * G + rows - 1) / rows);
  e.span = divide ? e.units : 1;
  return e;
}

// units of all of an entry's segments
__host__ __device__ __forceinline__ int64_t entry_work(const Entry& e, int kv_heads) {
  return (int64_t)e.span * e.tiles * kv_heads;
}

// floor(a / b) for 0 <= a < 2^52, b > 0, by a float64 quotient that is at most one off (a
// 64-bit integer division is a hundred and fifty instructions here)
__host__ __device__ __forceinline__ int64_t div_floor(int64_t a, int64_t b) {
  int64_t q = (int64_t)((double)a / (double)b);
  const int64_t r = a - q * b;
  if (r < 0) --q;
  if (r >= b) ++q;
  return q;
}

// first unit of workgroup i of n, of U units in all; the workgroup that has unit x
__host__ __device__ __forceinline__ int64_t first_unit(int i, int n, int64_t U) { return div_floor(U * i, n); }
__host__ __device__ __forceinline__ int owner(int64_t x, int n, int64_t U) { return (int)div_floor((x + 1) * n - 1, U); }

}  // namespace cattn
}  // namespace sva
