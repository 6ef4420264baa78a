// How the keys of a call are divided among workgroups (cache_attn_kernel.h,
// cache_attention.hip).  Host and device code, so that the division can be
// checked without a GPU.
//
// A segment is one (batch entry, cache head, row tile); its keys are cut into
// units of 128 (a 32-key step of each of four waves): first the cached keys,
// then the drafted ones, at least one unit.  The units of all segments, in the
// order (entry, head, tile, key), are dealt to n workgroups in runs of equal
// length: units have places (one each; where runs are long a segment's first takes
// kBegin more, for what beginning a segment costs), and workgroup i takes the units
// whose places begin in [i*W/n, (i+1)*W/n) of W.  However ragged the lengths, every
// workgroup then has the same work; a run may cross segments, and a segment whose
// units went to several workgroups is joined from their partial results afterwards.
// Short caches are not divided (their segments count as one unit each): joining would
// cost more than it gives.  A workgroup leaves at most two parts: slot 2i for a run that
// begins inside a segment, 2i + 1 for one that begins with a segment and ends inside it.
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

namespace sva {
namespace cattn {

constexpr int kUnit = 128;       // keys of a unit
// Segments of at most so many units are not divided: the join's launch takes longer than the
// units one after the other (us a call, divided / whole, 8 cache heads of 500 tokens: one
// sequence 18.4 / 15.6, 64 of them 25.7 / 19.7; 16 of 900 tokens 19.9 / 21.4, one of 1,900
// 17.6 / 30.6)
constexpr int kWholeUnits = 6;
constexpr int kWaves = 4;

// Workgroups per CU (waves per SIMD) of cache_attn_kernel with QT row tiles: at D = 64 and
// one tile a third finds its registers, and brings 943 MB from 102 us to 90; at D = 128 it
// would spill (137 us to 155 for 840 MB)
constexpr int wave_residents(int D, int QT) { return D == 64 && QT == 1 ? 3 : 2; }

// What beginning a segment costs, in units: its first loads are waited for, and its waves' results
// meet.  48 ragged sequences of 512 to 32,760 e4m3 tokens, us: none 176, one 167, two 162, four 165
constexpr int kBegin = 2;

struct Entry {                   // one batch entry
  int len;                       // cached tokens
  int cnt;                       // drafted tokens
  int cached_units, units;       // of each of its segments
  int tiles;                     // row tiles
  int begin;                     // places that beginning a segment takes; < 0: segments are not divided
  int span;                      // places of a segment
};

__host__ __device__ __forceinline__ Entry entry_of(int len, int cnt, int max_len, int T, int G, int rows, bool drafts,
                                                         int begin) {
  Entry e;
  e.len = len < 0 ? 0 : (len > max_len ? max_len : len);
  e.cnt = cnt < 0 ? 0 : (cnt > T ? T : cnt);
  e.cached_units = (int)(((int64_t)e.len + kUnit - 1) / kUnit);
  e.units = e.cached_units + (drafts ? (e.cnt + kUnit - 1) / kUnit : 0);
  if (e.units < 1) e.units = 1;
  e.tiles = (e.cnt * G + rows - 1) / rows;   // (cnt <= 1,024, G <= 65,536)
  e.begin = begin;
  e.span = begin < 0 ? 1 : e.units + begin;
  return e;
}

// places of all of an entry's segments
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

// where workgroup i's run begins, of n and W places; the workgroup whose run holds place x
__host__ __device__ __forceinline__ int64_t run_of(int i, int n, int64_t W) { return div_floor(W * i, n); }
__host__ __device__ __forceinline__ int owner(int64_t x, int n, int64_t W) { return (int)div_floor((x + 1) * n - 1, W); }
// the places that beginning a segment takes in a call of U units on a grid: none where runs
// are short, so that each has a unit
__host__ __device__ __forceinline__ int begin_of(int64_t U, int grid) { return U >= (int64_t)8 * grid ? kBegin : 0; }

// The segment at place `off` of an entry (with work), and its units that begin in [off, off + run).
struct Piece {
  int seg;
  int u0, u1;                    // (none where u0 == u1: the run begins inside a last unit)
  int64_t next;                  // place behind them
};
__host__ __device__ __forceinline__ int units_before(const Entry& e, int64_t place) {
  const int64_t k = place <= 0 ? 0 : (place <= e.begin ? 1 : place - e.begin);
  return (int)(k < e.units ? k : e.units);
}
__host__ __device__ __forceinline__ Piece piece_at(const Entry& e, int64_t off, int64_t run) {
  Piece p;
  p.seg = (int)div_floor(off, e.span);
  const int64_t at = off - (int64_t)p.seg * e.span;
  if (e.begin < 0) {
    p.u0 = 0;
    p.u1 = e.units;
    p.next = off + 1;
  } else {
    p.u0 = units_before(e, at);
    p.u1 = units_before(e, at + run);
    p.next = at + run < e.span ? off + run : off - at + e.span;
  }
  return p;
}
// place of a segment's unit in its entry
__host__ __device__ __forceinline__ int64_t place_of(const Entry& e, int64_t seg, int unit) {
  return seg * e.span + (unit > 0 ? unit + e.begin : 0);
}

}  // namespace cattn
}  // namespace sva
