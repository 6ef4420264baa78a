// What the cross-attention kernels share: strided, gathered rows into LDS tiles
// that serve both as rows (ds_read_b128) and transposed (ds_read_b64_tr_b16).
#pragma once

#include "attn_w16.h"
#include "cross_args.h"

namespace sva {
namespace cross {

using namespace attn;

constexpr int kThreads = 256;    // four waves
constexpr int CK = 32;           // rows of a tile

// LDS position of 16-byte piece c of tile row r.  A b128 read takes one piece of 16
// consecutive rows, a transpose read pieces 2dt and 2dt + 1 of eight: both fall on
// all 64 banks where the XOR differs in its upper bits over eight rows (two of which
// share a bank window at a 128-byte pitch) and in its lowest between rows r and r + 8.
template <int NCH>
__device__ __forceinline__ int swz(int r, int c) {
  return NCH == 16 ? c ^ (((r & 7) << 1) | ((r >> 3) & 1)) : c ^ ((((r >> 1) & 3) << 1) | ((r >> 3) & 1));
}

// Per-lane LDS offsets of the row operand of step s (rows i; 16 rows further the
// swizzle is the same) and of the first transpose read of d tile dt.
template <int D>
__device__ __forceinline__ void operand_offsets(int lane, int (&koff)[Geo16<D>::KS], int (&voff)[Geo16<D>::DT]) {
  using G = Geo<D>;
  const int g = lane >> 4, i = lane & 15;
#pragma unroll
  for (int s = 0; s < Geo16<D>::KS; ++s) koff[s] = i * G::RB + (swz<G::NCH>(i, 4 * s + g) << 4);
  const int r1 = 4 * g + (i >> 2);
#pragma unroll
  for (int dt = 0; dt < Geo16<D>::DT; ++dt)
    voff[dt] = r1 * G::RB + (swz<G::NCH>(r1, 2 * dt + ((i & 3) >> 1)) << 4) + (i & 1) * 8;
}

// What rows that are not there and channels past D are loaded from.
__device__ const uint4 kZeros[16] = {};
__device__ const float kInf[2] = {INFINITY, 0.0f};   // a row's lse and delta

typedef __attribute__((address_space(1))) const void global_void;
typedef __attribute__((address_space(3))) void lds_void;

template <int BYTES>
__device__ __forceinline__ void global_to_lds(const void* from, unsigned lds_addr) {
  lds_void* to = (lds_void*)(size_t)__builtin_amdgcn_readfirstlane(lds_addr);
  if constexpr (BYTES == 16) __builtin_amdgcn_global_load_lds((global_void*)from, to, 16, 0, 0);
  else __builtin_amdgcn_global_load_lds((global_void*)from, to, 4, 0, 0);
}

// Direct global -> LDS loads of one tile of 32 rows: the NUW 1 KB pieces a wave
// fills.  Piece u covers tile rows u * RPI ..; lane L fills row u * RPI + L / NCH at
// position L % NCH with the piece that the swizzle maps there.
template <int D>
struct TileLoader {
  using G = Geo<D>;
  static constexpr int CT = CK * G::RB;          // bytes of a tile
  static constexpr int NUW = CT / 1024 / (kThreads / 64);
  int row[NUW], chan[NUW];                       // of the tile, element offset in the row (negative: padding)
  int w;

  __device__ __forceinline__ void init(int wave, int lane) {
    w = wave;
#pragma unroll
    for (int u = 0; u < NUW; ++u) {
      row[u] = (wave * NUW + u) * G::RPI + lane / G::NCH;
      const int c = swz<G::NCH>(row[u], lane % G::NCH);
      chan[u] = c < G::DCH ? c * 8 : -1;
    }
  }
  // rows first .. first + 31 of `count` behind `base`, row pitch `pitch` elements
  __device__ __forceinline__ void load(const uint16_t* base, int64_t pitch, int first, int count, unsigned lds) const {
    if (__builtin_expect(first + CK <= count, 1) && G::DCH == G::NCH) {
      const uint16_t* p = base + (int64_t)first * pitch;
#pragma unroll
      for (int u = 0; u < NUW; ++u) global_to_lds<16>(p + (row[u] * pitch + chan[u]), lds + (w * NUW + u) * 1024);
    } else {
#pragma unroll
      for (int u = 0; u < NUW; ++u) {
        const bool there = first + row[u] < count && chan[u] >= 0;
        const void* p = base + ((int64_t)first + row[u]) * pitch + chan[u];
        global_to_lds<16>(there ? p : (const void*)kZeros, lds + (w * NUW + u) * 1024);
      }
    }
  }
  // the rows that `list` (indexed by u) names, those from `valid` on being absent
  __device__ __forceinline__ void load_rows(const uint16_t* base, int64_t pitch, const int (&list)[NUW], int valid, unsigned lds) const {
#pragma unroll
    for (int u = 0; u < NUW; ++u) {
      const bool there = row[u] < valid && chan[u] >= 0;
      const void* p = base + list[u] * pitch + chan[u];
      global_to_lds<16>(there ? p : (const void*)kZeros, lds + (w * NUW + u) * 1024);
    }
  }
};

// keys of an entry that queries see
__device__ __forceinline__ int seen_keys(const CrossArgs& a, int b) {
  const int n = a.mask ? a.seen[b] : a.lens ? a.lens[b] : a.M;
  return min(max(n, 0), a.M);
}
// the same of a workgroup's one entry, as a scalar
__device__ __forceinline__ int seen_keys_of_all(const CrossArgs& a, int b) {
  int n = a.M;
  if (a.mask) n = ((const_i32*)a.seen)[b];
  else if (a.lens) n = ((const_i32*)a.lens)[b];
  return __builtin_amdgcn_readfirstlane(min(max(n, 0), a.M));
}

// Row r of a kv head's R rows is token r % N of the group's head r / N.
__device__ __forceinline__ int64_t row_offset(const HeadsView& t, int b, int head0, int r, int N) {
  const int g = r / N, n = r - g * N;
  return b * t.sb + (head0 + g) * t.sh + n * t.sn;
}

// B operands of rows base + qt * 16 + i at d = 32s + 8g .. +8; zeros for an absent row or d >= D
template <int D, int QT>
__device__ __forceinline__ void load_operand(bf16x8 (&op)[QT][Geo16<D>::KS], const uint16_t* const (&rows)[QT], int lane) {
  const int g = lane >> 4;
#pragma unroll
  for (int qt = 0; qt < QT; ++qt)
#pragma unroll
    for (int s = 0; s < Geo16<D>::KS; ++s) {
      const int d0 = s * 32 + g * 8;
      if (rows[qt] && d0 < D) op[qt][s] = *reinterpret_cast<const bf16x8*>(rows[qt] + d0);
      else op[qt][s] = bf16x8{};
    }
}

// The keys' places where a mask hides some: 1,024 entries of the list of seen keys in
// LDS, refilled 512 at a time while the others are in use.
struct RowRing {
  static constexpr int kSize = 1024, kHalf = 512;
  int* ring;
  const int32_t* list;
  int end;                       // of the list
  __device__ __forceinline__ void fill(int first) {
    for (int e = threadIdx.x; e < kHalf; e += kThreads) ring[(first + e) % kSize] = list[min(first + e, end - 1)];
  }
  __device__ __forceinline__ int at(int key) const { return ring[key % kSize]; }
};

}  // namespace cross
}  // namespace sva
