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

typedef __attribute__((address_space(3))) const bf16x8 lds_bf16x8;

// Workgroups of 32 rows a wave that a CU holds: two, whose waves have 256 registers each.
// Heads of 64 fit the 168 of three: 31,620 tokens' 40 heads over 512 keys take 260 us
// instead of 305, their gradients 880 instead of 920.
constexpr int wide_per_cu(int D) { return D == 64 ? 3 : 2; }

// A lane's place in a tile, for the row operands (row i at channels 8g .. +8) and for the
// transpose reads (rows 4g.. at channels 0..).  Step s of the rows is at place ^ s << 6,
// d tile dt at place ^ dt << 5, 16 rows further the swizzle is the same: one register
// holds them all.
template <int D>
struct Places {
  unsigned row, col;
  __device__ __forceinline__ explicit Places(int lane) {
    using G = Geo<D>;
    const int g = lane >> 4, i = lane & 15, r1 = 4 * g + (i >> 2);
    row = i * G::RB + (swz<G::NCH>(i, g) << 4);
    col = r1 * G::RB + (swz<G::NCH>(r1, (i & 3) >> 1) << 4) + (i & 1) * 8;
  }
};

// S = 16 of a tile's rows, the first at LDS address `tile`, times the rows in registers:
// for the tile's rows 4g + r and the register rows 16qt + i, sum over d
template <int D, int QT>
__device__ __forceinline__ void rows_times_half(f32x4 (&s)[QT], unsigned tile, const Places<D>& at,
                                                const bf16x8 (&op)[QT][Geo16<D>::KS]) {
  const unsigned p = tile + at.row;
#pragma unroll
  for (int qt = 0; qt < QT; ++qt) s[qt] = f32x4{};
#pragma unroll
  for (int k = 0; k < Geo16<D>::KS; ++k) {
    const bf16x8 row = *(lds_bf16x8*)(size_t)(p ^ (k << 6));
#pragma unroll
    for (int qt = 0; qt < QT; ++qt) s[qt] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(row, op[qt][k], s[qt], 0, 0, 0);
  }
}

// Eight wait states between products and whatever reads them: vector instructions may read a
// product so much after its last instruction, and where a branch comes between, the compiler has
// left them out.
template <int QT>
__device__ __forceinline__ void settle(f32x4 (&x)[QT], f32x4 (&y)[QT]) {
  if constexpr (QT == 1) asm volatile("s_nop 7" : "+v"(x[0]), "+v"(y[0]));
  else asm volatile("s_nop 7" : "+v"(x[0]), "+v"(x[1]), "+v"(y[0]), "+v"(y[1]));
}

// acc += the tile's columns times the weights in registers, over its 32 rows in the order
// of attn_w16.h
template <int D, int QT>
__device__ __forceinline__ void cols_times(const bf16x8 (&wop)[QT], unsigned tile, const Places<D>& at,
                                           f32x4 (&acc)[Geo16<D>::DT][QT]) {
  using G = Geo<D>;
  const unsigned p = tile + at.col;
#pragma unroll
  for (int dt = 0; dt < Geo16<D>::DT; ++dt) {
    const unsigned q = p ^ (dt << 5);
    const u32x2 lw = __builtin_bit_cast(u32x2, __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_i16x4*)(size_t)q));
    const u32x2 hw = __builtin_bit_cast(u32x2, __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_i16x4*)(size_t)(q + 16 * G::RB)));
    const bf16x8 col = __builtin_bit_cast(bf16x8, u32x4{lw[0], lw[1], hw[0], hw[1]});
#pragma unroll
    for (int qt = 0; qt < QT; ++qt) acc[dt][qt] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(col, wop[qt], acc[dt][qt], 0, 0, 0);
  }
}

// The same with two sets of weights.
template <int D, int QT>
__device__ __forceinline__ void cols_times_both(const bf16x8 (&w0)[QT], const bf16x8 (&w1)[QT], unsigned tile, const Places<D>& at,
                                                f32x4 (&acc0)[Geo16<D>::DT][QT], f32x4 (&acc1)[Geo16<D>::DT][QT]) {
  using G = Geo<D>;
  const unsigned p = tile + at.col;
#pragma unroll
  for (int dt = 0; dt < Geo16<D>::DT; ++dt) {
    const unsigned q = p ^ (dt << 5);
    const u32x2 lw = __builtin_bit_cast(u32x2, __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_i16x4*)(size_t)q));
    const u32x2 hw = __builtin_bit_cast(u32x2, __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_i16x4*)(size_t)(q + 16 * G::RB)));
    const bf16x8 col = __builtin_bit_cast(bf16x8, u32x4{lw[0], lw[1], hw[0], hw[1]});
#pragma unroll
    for (int qt = 0; qt < QT; ++qt) {
      acc0[dt][qt] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(col, w0[qt], acc0[dt][qt], 0, 0, 0);
      acc1[dt][qt] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(col, w1[qt], acc1[dt][qt], 0, 0, 0);
    }
  }
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
// position L % NCH with the piece that the swizzle maps there.  A pitch of D = 112 leaves
// two positions of a row without a piece: those lanes load nothing, and what is there is
// cleared once.
template <int D>
struct TileLoader {
  using G = Geo<D>;
  static constexpr int CT = CK * G::RB;          // bytes of a tile
  static constexpr int NUW = CT / 1024 / (kThreads / 64);
  static constexpr bool PAD = G::DCH != G::NCH;
  int w, lane;

  __device__ __forceinline__ void init(int wave, int ln) {
    w = wave;
    lane = ln;
  }
  __device__ __forceinline__ int row(int u) const { return (w * NUW + u) * G::RPI + lane / G::NCH; }
  __device__ __forceinline__ int piece(int u) const { return swz<G::NCH>(row(u), lane % G::NCH); }
  // zeros where no piece goes, in `stages` tiles from `tiles` on
  __device__ __forceinline__ void clear_pads(unsigned char* tiles, int stages) const {
    if constexpr (PAD) {
#pragma unroll
      for (int u = 0; u < NUW; ++u)
        if (piece(u) >= G::DCH)
          for (int st = 0; st < stages; ++st) *reinterpret_cast<u32x4*>(tiles + st * CT + (w * NUW + u) * 1024 + lane * 16) = u32x4{};
    }
  }
  // byte offsets of the lane's pieces from a tile's first row, where they fit in 32 bits
  static __device__ __forceinline__ bool near(int64_t pitch) { return pitch < (int64_t)1 << 25; }
  __device__ __forceinline__ void offsets(int64_t pitch, uint32_t (&off)[NUW]) const {
#pragma unroll
    for (int u = 0; u < NUW; ++u) off[u] = near(pitch) ? (uint32_t)(row(u) * (int)pitch + piece(u) * 8) * 2u : 0u;
  }
  // a whole tile whose first row is at `tile`
  __device__ __forceinline__ void load_near(const uint16_t* tile, const uint32_t (&off)[NUW], unsigned lds) const {
#pragma unroll
    for (int u = 0; u < NUW; ++u)
      if (!PAD || piece(u) < G::DCH)
        global_to_lds<16>(reinterpret_cast<const unsigned char*>(tile) + off[u], lds + (w * NUW + u) * 1024);
  }
  // the rows of a tile whose bits are set, zeros in place of the others
  __device__ __forceinline__ void load_some(const uint16_t* tile, int64_t pitch, uint32_t bits, unsigned lds) const {
    // The lane id goes through an empty asm, so that what this rarer path needs is worked
    // out here and not kept in registers.
    int ln = lane;
    asm volatile("" : "+v"(ln));
#pragma unroll
    for (int u = 0; u < NUW; ++u) {
      const int r = (w * NUW + u) * G::RPI + ln / G::NCH, c = swz<G::NCH>(r, ln % G::NCH);
      if (!PAD || c < G::DCH) {
        const void* p = tile + (int64_t)r * pitch + c * 8;
        global_to_lds<16>(bits >> r & 1 ? p : (const void*)kZeros, lds + (w * NUW + u) * 1024);
      }
    }
  }
  // the same by the near offsets, for masks with holes
  __device__ __forceinline__ void load_some_near(const uint16_t* tile, const uint32_t (&off)[NUW], uint32_t bits, unsigned lds) const {
    const uint32_t mine = bits >> row(0);
#pragma unroll
    for (int u = 0; u < NUW; ++u)
      if (!PAD || piece(u) < G::DCH) {
        const void* p = reinterpret_cast<const unsigned char*>(tile) + off[u];
        global_to_lds<16>(mine >> (u * G::RPI) & 1 ? p : (const void*)kZeros, lds + (w * NUW + u) * 1024);
      }
  }
  template <bool HOLES = false>
  __device__ __forceinline__ void load(const uint16_t* tile, int64_t pitch, const uint32_t (&off)[NUW], uint32_t bits, unsigned lds) const {
    if (__builtin_expect(bits == ~0u && near(pitch), 1)) load_near(tile, off, lds);
    else if (HOLES && near(pitch)) load_some_near(tile, off, bits, lds);
    else load_some(tile, pitch, bits, lds);
  }
};

// Which of a tile's 32 rows are there, `left` of them or more being left.
__device__ __forceinline__ uint32_t rows_left(int left) { return left >= CK ? ~0u : left > 0 ? (1u << left) - 1u : 0u; }

// keys of an entry up to the last that queries see
__device__ __forceinline__ int seen_keys(const CrossArgs& a, int b) {
  const int n = a.mask ? a.seen[b] : a.lens ? a.lens[b] : a.M;
  return min(max(n, 0), a.M);
}
// whether queries see key m, one of the entry's `count` first
__device__ __forceinline__ bool is_seen(const CrossArgs& a, int b, int m, int count) {
  return m < count && (!a.mask || (a.bits[(int64_t)b * ((a.M + 31) / 32) + m / 32] >> (m % 32) & 1));
}
// the same of a workgroup's one entry, as a scalar
__device__ __forceinline__ int seen_keys_of_all(const CrossArgs& a, int b) {
  int n = a.M;
  if (a.mask) n = ((const_i32*)a.seen)[b];
  else if (a.lens) n = ((const_i32*)a.lens)[b];
  return __builtin_amdgcn_readfirstlane(min(max(n, 0), a.M));
}

// Row r of a kv head's R rows is token r % N of the group's head r / N.
__device__ __forceinline__ int64_t row_offset(const HeadsView& t, int b, int head0, int r, int N, int G) {
  int g = 0;
  if (G > 1) g = r / N;
  return b * t.sb + (head0 + g) * t.sh + (int64_t)(r - g * N) * t.sn;
}

// B operands of rows base + qt * 16 + i at d = 32s + 8g .. +8; zeros for an absent row (null)
// or d >= D, loaded like the others, so that every call issues as many loads
template <int D, int QT>
__device__ __forceinline__ void load_operand(bf16x8 (&op)[QT][Geo16<D>::KS], const uint16_t* const (&rows)[QT], int lane) {
  const int g = lane >> 4;
#pragma unroll
  for (int qt = 0; qt < QT; ++qt) {
    const uint16_t* row = rows[qt] ? rows[qt] : reinterpret_cast<const uint16_t*>(kZeros);
#pragma unroll
    for (int s = 0; s < Geo16<D>::KS; ++s) {
      const int d0 = s * 32 + g * 8;
      const uint16_t* p = D % 32 == 0 || d0 < D ? row + d0 : reinterpret_cast<const uint16_t*>(kZeros);
      op[qt][s] = *reinterpret_cast<const bf16x8*>(p);
    }
  }
}

// A workgroup's work: some row tiles of a kv head, one after the other, against its keys,
// or one against a part of them.  Kv heads are the fastest of the three, so that the heads
// of a token, which lie together in a projection's output, are read at about the same
// time, and an XCD (every eighth workgroup) has few heads' keys in its L2.
struct Item {
  int b, kvh, split, tile, tiles;
  int count, c0, chunks;         // keys that the entry has, the first 32-key tile and how many

  __device__ __forceinline__ explicit Item(const CrossArgs& a) {
    const int heads = a.B * a.Hkv, part = blockIdx.x / heads, bh = blockIdx.x - part * heads;
    const int groups = (a.tiles + a.run - 1) / a.run;
    split = part / groups;
    tile = (part - split * groups) * a.run;
    tiles = min(a.run, a.tiles - tile);
    b = bh / a.Hkv;
    kvh = bh - b * a.Hkv;
    count = seen_keys_of_all(a, b);
    chunks = (count + CK - 1) / CK;
    c0 = 0;
    if (a.splits > 1) {
      c0 = (int)((int64_t)chunks * split / a.splits);
      chunks = (int)((int64_t)chunks * (split + 1) / a.splits) - c0;
    }
  }
};

// Feeds tiles of K and V to a workgroup, over and over for one row tile after the other,
// and says which of a tile's keys are seen: with a mask, a word of `bits` for each tile,
// read a step ahead as a scalar.  KEYS_TOO: zeros in place of hidden rows of K as of V.
template <int D, bool MASK, bool KEYS_TOO>
struct KeyFeed {
  using Loader = TileLoader<D>;
  static constexpr int NUW = Loader::NUW;
  static constexpr int kLoads = 2 * NUW;         // of a wave for a tile
  Loader ld;
  const uint16_t *k0, *v0, *kp, *vp;             // the first tile's first row, and the next one's
  int keys, left;                                // keys of the part, and from the next tile on
  uint32_t koff[NUW], voff[NUW];
  const uint32_t *words0, *words;                // MASK
  uint32_t word;

  __device__ __forceinline__ void look_up() {
    if constexpr (MASK) word = *(const __attribute__((address_space(4))) uint32_t*)words;
    else word = rows_left(left);
  }
  __device__ __forceinline__ void rewind() {
    kp = k0;
    vp = v0;
    left = keys;
    if constexpr (MASK) words = words0;
  }
  // (the part has a key)
  __device__ __forceinline__ void start(const CrossArgs& a, const Item& it, int w, int lane) {
    ld.init(w, lane);
    const int64_t row = (int64_t)it.c0 * CK;
    k0 = static_cast<const uint16_t*>(a.k.p) + it.b * a.k.sb + it.kvh * a.k.sh + row * a.k.sn;
    v0 = static_cast<const uint16_t*>(a.v.p) + it.b * a.v.sb + it.kvh * a.v.sh + row * a.v.sn;
    // keys of the next part are not there
    keys = min(it.count - it.c0 * CK, it.chunks * CK);
    if constexpr (MASK) words0 = a.bits + (int64_t)it.b * ((a.M + 31) / 32) + it.c0;
    rewind();
    look_up();
    ld.offsets(a.k.sn, koff);
    ld.offsets(a.v.sn, voff);
  }
  // the next tile into LDS, after the last one the first; returns which of its keys are seen
  __device__ __forceinline__ uint32_t feed(const CrossArgs& a, unsigned ks, unsigned vs) {
    const uint32_t now = __builtin_amdgcn_readfirstlane(word);
    // hidden keys of a mask are read where their logits alone are formed (and replaced)
    ld.template load<MASK && KEYS_TOO>(kp, a.k.sn, koff, MASK && !KEYS_TOO ? rows_left(left) : now, ks);
    ld.template load<MASK>(vp, a.v.sn, voff, now, vs);
    kp += CK * a.k.sn;
    vp += CK * a.v.sn;
    left -= CK;
    if constexpr (MASK) ++words;
    if (left <= 0) rewind();
    look_up();
    return now;
  }
};

// A row's D channels to memory as bf16, f times what the lanes hold: lane (g, i) has channels
// 16dt + 4g .. +4 of row i of a 16-row tile.  Neighbours in g first trade halves of two d
// tiles, so that a lane writes 16 bytes and four lanes 64 in a row: in 8-byte pieces of 32
// in a row, 63,240 tokens of 32 heads of 128 over 128 keys took 330 us, so 286.
template <int D>
__device__ __forceinline__ void store_row(uint16_t* row, const f32x4* acc, int stride, float f, int g) {
  constexpr int DT = D / 16;
#pragma unroll
  for (int dt = 0; dt < DT; dt += 2) {
    const f32x4 x = acc[dt * stride];
    const bf16x2 x0 = cvt2(x[0] * f, x[1] * f), x1 = cvt2(x[2] * f, x[3] * f);
    if (dt + 1 < DT) {
      const f32x4 y = acc[(dt + 1) * stride];
      const bf16x2 y0 = cvt2(y[0] * f, y[1] * f), y1 = cvt2(y[2] * f, y[3] * f);
      const u32x2 lo = __builtin_amdgcn_permlane16_swap(__builtin_bit_cast(unsigned, x0), __builtin_bit_cast(unsigned, y0), false, false);
      const u32x2 hi = __builtin_amdgcn_permlane16_swap(__builtin_bit_cast(unsigned, x1), __builtin_bit_cast(unsigned, y1), false, false);
      // even g: channels 16dt + 4g .. +8, odd g: 16(dt + 1) + 4(g - 1) .. +8
      if (row) *reinterpret_cast<u32x4*>(row + (dt + (g & 1)) * 16 + 4 * (g & 2)) = u32x4{lo[0], hi[0], lo[1], hi[1]};
    } else if (row) {
      const bf16x4 z = {x0[0], x0[1], x1[0], x1[1]};
      *reinterpret_cast<bf16x4*>(row + dt * 16 + 4 * g) = z;
    }
  }
}

// logits of a tile's hidden keys to -inf
template <int QT>
__device__ __forceinline__ void hide(f32x4 (&s)[2][QT], uint32_t bits, int lane) {
  const uint32_t mine = bits >> (4 * (lane >> 4));
#pragma unroll
  for (int k2 = 0; k2 < 2; ++k2)
#pragma unroll
    for (int r = 0; r < 4; ++r)
      if (!(mine >> (k2 * 16 + r) & 1)) {
#pragma unroll
        for (int qt = 0; qt < QT; ++qt) s[k2][qt][r] = -INFINITY;
      }
}

}  // namespace cross
}  // namespace sva
