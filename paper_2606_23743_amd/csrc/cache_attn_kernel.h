// Attention of drafted tokens over a paged cache: softmax(c Q K^T) V for the
// G * T query rows that share one cache head (row = t * G + g), keys read once
// per tile of up to 64 rows.
//
// What bounds it: with one token the keys and values come from HBM once and each
// code meets at most 16 rows, so it is bound by HBM; from about 64 rows on the
// products and the softmax take as long.  So the shape is: every wave walks 32-key
// steps of its own with its own running maximum and sum, straight from memory into
// registers (no barrier and no LDS in the loop, whatever the page order), and the
// waves meet once per segment in LDS.  The division of keys among workgroups is
// in cache_attn_plan.h.
//
// Lane l = 16g + i.  One step, 32 keys, on mfma_f32_16x16x32_bf16:
//   S^T tile x (x = 0, 1) = K Q^T: A operand row m is key 8(m/4) + 4x + m%4, so
//     that the result leaves lane (g, i) with keys 8g + 4x + 0..3 of query column
//     i: over both tiles the eight consecutive keys 8g .. 8g + 7.  The channels of
//     step s are 32s + 8g .. + 7 (bf16 cache) or 64(s/2) + 16g + 8(s%2) .. + 7 (8 bits:
//     one 16-byte piece of a row feeds two steps); Q is laid out alike.
//   P^T of those eight keys is, in this order, the B operand of
//   O^T tile j += V^T P^T, whose A operand is row r = channel JT * r + j at the
//     eight keys 8g .. 8g + 7: a lane loads JT consecutive channels of each of
//     eight rows and transposes in registers (byte permutes), so V needs no LDS
//     either, and a result lane holds JT consecutive channels per register row.
// 8-bit codes are widened to bf16 exactly (e4m3 has 4 significant bits, int8 at
// most 7 and a sign); a token's K scale multiplies its logits, its V scale its weights,
// in float32.
//
// The running maximum moves only where a step's logits pass it by more than 8 (in
// base 2): weights stay below 2^8 and most steps rescale nothing.
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

template <int FMT, int D>
struct CGeo {
  static constexpr bool W8 = FMT != kCacheBf16;
  static constexpr int EB = W8 ? 1 : 2;            // bytes of a code
  static constexpr int KS = D > 64 ? 4 : 2;        // 32-channel steps of the S products
  static constexpr int NPK = KS * EB / 2 > 0 ? KS * EB / 2 : 1;   // 16-byte pieces of a K row per lane
  static constexpr int JT = D > 64 ? 8 : 4;        // channels of a V row per lane = O^T tiles
  static constexpr int VR = D / JT;                // lanes of a V row that hold channels (16, or 14 at D = 112)
  static constexpr int NW = JT * EB / 4;           // dwords of a V row per lane
};

// first channel of step s in lane group g
template <bool W8>
__device__ __forceinline__ int chan(int s, int g) { return W8 ? 64 * (s >> 1) + 16 * g + 8 * (s & 1) : 32 * s + 8 * g; }

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

// the raw K and V of one 32-key step
template <int FMT, int D>
struct Raw {
  using G = CGeo<FMT, D>;
  u32x4 k[2][G::NPK];
  uint32_t v[8][G::NW];
};

// V^T operand of tile j: channel JT * r + j of keys 8g .. 8g + 7.  8-bit codes are
// transposed four channels at a time (t: the bytes of keys 0..3 and 4..7 of each).
template <int NW>
__device__ __forceinline__ bf16x8 v_operand16(const uint32_t (&v)[8][NW], int j) {
  u32x4 o;
  const uint32_t sel = (j & 1) ? 0x07060302u : 0x05040100u;
#pragma unroll
  for (int p = 0; p < 4; ++p) o[p] = __builtin_amdgcn_perm(v[2 * p + 1][j >> 1], v[2 * p][j >> 1], sel);
  return __builtin_bit_cast(bf16x8, o);
}
template <int NW>
__device__ __forceinline__ void transpose8(const uint32_t (&v)[8][NW], int w, uint32_t (&t)[4][2]) {
#pragma unroll
  for (int h = 0; h < 2; ++h) {
    const uint32_t a = v[4 * h][w], b = v[4 * h + 1][w], c = v[4 * h + 2][w], d = v[4 * h + 3][w];
    const uint32_t ab0 = __builtin_amdgcn_perm(b, a, 0x05010400u), ab1 = __builtin_amdgcn_perm(b, a, 0x07030602u);
    const uint32_t cd0 = __builtin_amdgcn_perm(d, c, 0x05010400u), cd1 = __builtin_amdgcn_perm(d, c, 0x07030602u);
    t[0][h] = __builtin_amdgcn_perm(cd0, ab0, 0x05040100u);
    t[1][h] = __builtin_amdgcn_perm(cd0, ab0, 0x07060302u);
    t[2][h] = __builtin_amdgcn_perm(cd1, ab1, 0x05040100u);
    t[3][h] = __builtin_amdgcn_perm(cd1, ab1, 0x07060302u);
  }
}

// one wave's running state for QT tiles of 16 rows
template <int D, int QT>
struct State {
  static constexpr int JT = D > 64 ? 8 : 4;
  f32x4 o[JT][QT];
  float m[QT], l[QT];            // reference (base 2) of the lane's column; the lane's part of the sum

  __device__ __forceinline__ void clear() {
#pragma unroll
    for (int qt = 0; qt < QT; ++qt) {
      m[qt] = -INFINITY;
      l[qt] = 0.0f;
#pragma unroll
      for (int j = 0; j < JT; ++j) o[j][qt] = f32x4{};
    }
  }

  // logits (base 2, -inf where masked) -> weights in place; the reference moves up
  // where a column passes it by 8
  __device__ __forceinline__ void weigh(float (&s)[QT][8]) {
    bool grow = false;
    float top[QT];
#pragma unroll
    for (int qt = 0; qt < QT; ++qt) {
      top[qt] = s[qt][0];
#pragma unroll
      for (int e = 1; e < 8; ++e) top[qt] = fmaxf(top[qt], s[qt][e]);
      grow |= top[qt] > m[qt] + 8.0f;
    }
    if (__builtin_amdgcn_ballot_w64(grow) != 0) {
#pragma unroll
      for (int qt = 0; qt < QT; ++qt) {
        const float to = fmaxf(m[qt], attn::quad_max(top[qt]));
        const float f = to == -INFINITY ? 1.0f : __builtin_amdgcn_exp2f(m[qt] - to);
        m[qt] = to;
        l[qt] *= f;
#pragma unroll
        for (int j = 0; j < JT; ++j)
#pragma unroll
          for (int r = 0; r < 4; ++r) o[j][qt][r] *= f;
      }
    }
#pragma unroll
    for (int qt = 0; qt < QT; ++qt) {
      const float ref = m[qt] == -INFINITY ? 0.0f : m[qt];   // only masked keys so far: weights of zero
      float sum = 0.0f;
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        s[qt][e] = __builtin_amdgcn_exp2f(s[qt][e] - ref);
        sum += s[qt][e];
      }
      l[qt] += sum;
    }
  }
};

// weights times V scales as B operands: rounded to bf16, and with LOW the rounding's
// remainder as a second operand (float32 results)
template <int QT, bool LOW>
__device__ __forceinline__ void weight_operands(const float (&p)[QT][8], bf16x8 (&hi)[QT], bf16x8 (&lo)[QT]) {
#pragma unroll
  for (int qt = 0; qt < QT; ++qt) {
    u32x4 h, r;
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      const float a = p[qt][2 * e], b = p[qt][2 * e + 1];
      h[e] = __builtin_bit_cast(uint32_t, attn::cvt2(a, b));
      if constexpr (LOW)
        r[e] = __builtin_bit_cast(uint32_t, attn::cvt2(a - __uint_as_float(h[e] << 16),
                                                       b - __uint_as_float(h[e] & 0xFFFF0000u)));
    }
    hi[qt] = __builtin_bit_cast(bf16x8, h);
    if constexpr (LOW) lo[qt] = __builtin_bit_cast(bf16x8, r);
  }
}

template <int D, int QT, bool LOW>
__device__ __forceinline__ void pv_tile(State<D, QT>& st, int j, bf16x8 v, const bf16x8 (&hi)[QT],
                                        const bf16x8 (&lo)[QT]) {
#pragma unroll
  for (int qt = 0; qt < QT; ++qt) {
    st.o[j][qt] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(v, hi[qt], st.o[j][qt], 0, 0, 0);
    if constexpr (LOW) st.o[j][qt] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(v, lo[qt], st.o[j][qt], 0, 0, 0);
  }
}

// units of all segments, and the entry that unit x falls into with its first unit; by one wave
struct Finder {
  const CacheAttnArgs& a;
  int rows;
  int64_t incl;                  // B <= 64: the scan of the only chunk
  int64_t total;

  __device__ __forceinline__ Entry at(int b) const {
    return entry_of(a.lens[b], a.counts ? a.counts[b] : a.T, a.max_pages << a.c.log2_page, a.T, a.G, rows,
                    a.kn.p != nullptr);
  }
  __device__ __forceinline__ int64_t scan(int b0) const {
    const int b = b0 + (int)(threadIdx.x & 63);
    int64_t x = b < a.B ? entry_work(at(b), a.c.heads) : 0;
#pragma unroll
    for (int d = 1; d < 64; d *= 2) {
      const int64_t y = __shfl_up(x, d);
      if ((int)(threadIdx.x & 63) >= d) x += y;
    }
    return x;
  }
  __device__ __forceinline__ Finder(const CacheAttnArgs& args, int rows_) : a(args), rows(rows_) {
    total = 0;
    for (int b0 = 0; b0 < a.B; b0 += 64) {
      incl = scan(b0);
      total += __shfl(incl, 63);
    }
  }
  // x < total
  __device__ __forceinline__ int find(int64_t x, int64_t& first) const {
    int64_t base = 0;
    for (int b0 = 0;; b0 += 64) {
      const int64_t in = a.B <= 64 ? incl : scan(b0);
      const uint64_t past = __builtin_amdgcn_ballot_w64(base + in > x);
      if (past != 0) {
        const int k = __builtin_ctzll(past);
        first = base + (k > 0 ? __shfl(in, k > 0 ? k - 1 : 0) : 0);
        return __builtin_amdgcn_readfirstlane(b0 + k);
      }
      base += __shfl(in, 63);
    }
  }
};

// float values of a partial result: QT * 16 rows of 16 * JT channels, their references and sums
template <int D, int QT>
struct Part {
  static constexpr int JT = D > 64 ? 8 : 4;
  static constexpr int kRows = 16 * QT;
  static constexpr int kFloats = kRows * (16 * JT + 2);
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

template <int FMT, int D, int QT, bool LOW>
__global__ __launch_bounds__(256) __attribute__((amdgpu_waves_per_eu(QT == 4 ? 1 : 2)))
void cache_attn_kernel(CacheAttnArgs a) {
  using G = CGeo<FMT, D>;
  using S = State<D, QT>;
  using PT = Part<D, QT>;
  constexpr int JT = G::JT, KS = G::KS, RPT = 16 * QT;
  __shared__ __attribute__((aligned(16))) float so[kWaves][4][64][JT];   // one 16-row tile of each wave
  __shared__ float sm[kWaves][RPT], sl[kWaves][RPT];

  const int lane = threadIdx.x & 63, g = lane >> 4, i16 = lane & 15;
  const int w = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const bool drafts = a.kn.p != nullptr;
  const int log2p = a.c.log2_page, pmask = (1 << log2p) - 1;
  const int Hkv = a.c.heads;

  const Finder fd(a, RPT);
  const int64_t U = fd.total;
  if (U == 0) return;
  const int n = (int)min((int64_t)gridDim.x, U);
  // neighbouring runs on one XCD where row tiles of a head read the same keys; a grid
  // with workgroups to spare spreads over all XCDs instead
  const int me = a.G * a.T > RPT && n == (int)gridDim.x ? xcd_remap(blockIdx.x, n) : blockIdx.x;
  if (me >= n) return;
  int64_t x = first_unit(me, n, U);
  const int64_t end = first_unit(me + 1, n, U);
  int64_t ebase;                                   // first unit of entry b
  int b = fd.find(x, ebase);

  while (x < end) {
    const Entry en = fd.at(b);
    const int64_t work = entry_work(en, Hkv);
    if (x >= ebase + work) {                       // the next entry
      ebase += work;
      ++b;
      continue;
    }
    const int seg = (int)((x - ebase) / en.units);
    const int u0 = (int)(x - ebase - (int64_t)seg * en.units);
    const int u1 = (int)min((int64_t)en.units, u0 + (end - x));
    const int h = seg / en.tiles, rt = seg - h * en.tiles;
    x += u1 - u0;

    // ---- Q of this tile's rows ----
    bf16x8 q[QT][KS];
    int tok[QT], head[QT];                         // of the lane's column; tok = -1: no such row
#pragma unroll
    for (int qt = 0; qt < QT; ++qt) {
      const int row = rt * RPT + qt * 16 + i16;
      const int t = row / a.G;
      tok[qt] = t < en.cnt ? t : -1;
      head[qt] = h * a.G + (row - t * a.G);
      const uint16_t* p = static_cast<const uint16_t*>(a.q.p) + b * a.q.sb + head[qt] * a.q.sh + t * a.q.sn;
#pragma unroll
      for (int s = 0; s < KS; ++s) {
        const int d = chan<G::W8>(s, g);
        if (tok[qt] >= 0 && d < D) q[qt][s] = *reinterpret_cast<const bf16x8*>(p + d);
        else q[qt][s] = bf16x8{};
      }
    }

    S st;
    st.clear();

    // ---- cached keys ----
    const int32_t* table = a.table + (int64_t)b * a.max_pages;
    const int kq = 8 * (i16 >> 2), kv8 = 8 * g;    // this lane's K rows and V rows of a step begin here
    auto page_at = [&](int key) { return table[min(key >> log2p, a.max_pages - 1)]; };
    int pk = 0, pv = 0;
    const int ulast = min(u1, en.cached_units);
    if (u0 < ulast) {
      pk = page_at(u0 * kUnit + 32 * w + kq);
      pv = page_at(u0 * kUnit + 32 * w + kv8);
    }
    for (int u = u0; u < ulast; ++u) {
      const int key0 = u * kUnit + 32 * w;
      if (key0 >= en.len) break;                   // only in a sequence's last unit
      const bool there = pv >= 0 && pv < a.c.num_pages;
      const int64_t gk = pk >= 0 && pk < a.c.num_pages ? pk : 0, gv = there ? pv : 0;
      const int64_t rk = ((gk * Hkv + h) << log2p) + ((key0 + kq) & pmask) + (i16 & 3);
      const int64_t rv = ((gv * Hkv + h) << log2p) + ((key0 + kv8) & pmask);
      Raw<FMT, D> r;
      const uint8_t* kp = static_cast<const uint8_t*>(a.c.k) + rk * (D * G::EB);
      const uint8_t* vp = static_cast<const uint8_t*>(a.c.v) + rv * (D * G::EB);
      // D = 112: groups past the row's end read its last piece, and drop it below
      auto piece = [&](int p) { return min(64 * p + 16 * g, D * G::EB - 16); };
#pragma unroll
      for (int t = 0; t < 2; ++t)
#pragma unroll
        for (int p = 0; p < G::NPK; ++p)
          r.k[t][p] = *reinterpret_cast<const u32x4*>(kp + t * 4 * D * G::EB + piece(p));
      const int vat = min(i16, G::VR - 1) * JT * G::EB;
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        const uint8_t* p = vp + e * D * G::EB + vat;
        if constexpr (G::NW == 1) {
          r.v[e][0] = *reinterpret_cast<const uint32_t*>(p);
        } else if constexpr (G::NW == 2) {
          const uint2 y = *reinterpret_cast<const uint2*>(p);
          r.v[e][0] = y.x;
          r.v[e][1] = y.y;
        } else {
          const uint4 y = *reinterpret_cast<const uint4*>(p);
          r.v[e][0] = y.x;
          r.v[e][1] = y.y;
          r.v[e][2] = y.z;
          r.v[e][3] = y.w;
        }
      }
      float ks[8], vs[8];
      if constexpr (G::W8) {
#pragma unroll
        for (int e = 0; e < 8; e += 4) {
          const float4 y = *reinterpret_cast<const float4*>(a.c.ks + rv + e);
          const float4 z = *reinterpret_cast<const float4*>(a.c.vs + rv + e);
          ks[e] = y.x; ks[e + 1] = y.y; ks[e + 2] = y.z; ks[e + 3] = y.w;
          vs[e] = z.x; vs[e + 1] = z.y; vs[e + 2] = z.z; vs[e + 3] = z.w;
        }
      }
      if (u + 1 < ulast) {
        pk = page_at(key0 + kUnit + kq);
        pv = page_at(key0 + kUnit + kv8);
      }
      // keys that take part: all but in a sequence's last step or on a bad page
      int valid = 0xff;
      const bool whole = key0 + 32 <= en.len && __builtin_amdgcn_ballot_w64(!there) == 0;
      if (!whole) {
        const int left = en.len - key0 - kv8;
        valid = there ? (left >= 8 ? 0xff : (left > 0 ? (1 << left) - 1 : 0)) : 0;
#pragma unroll
        for (int e = 0; e < 8; ++e)
          if (!(valid >> e & 1)) {
            vs[e] = 0.0f;
#pragma unroll
            for (int d = 0; d < G::NW; ++d) r.v[e][d] = 0;
          }
      }
      f32x4 acc[2][QT];
#pragma unroll
      for (int t = 0; t < 2; ++t)
#pragma unroll
        for (int qt = 0; qt < QT; ++qt) acc[t][qt] = f32x4{};
#pragma unroll
      for (int s = 0; s < KS; ++s)
#pragma unroll
        for (int t = 0; t < 2; ++t) {
          u32x4 kw;
          if constexpr (G::W8) {
            const u32x2 y = widen4<FMT>(r.k[t][s >> 1][2 * (s & 1)]), z = widen4<FMT>(r.k[t][s >> 1][2 * (s & 1) + 1]);
            kw = u32x4{y[0], y[1], z[0], z[1]};
          } else {
            kw = r.k[t][s];
          }
          if (D == 112 && chan<G::W8>(s, 3) >= D) {  // a step with absent channels
            if (chan<G::W8>(s, g) >= D) kw = u32x4{};
          }
#pragma unroll
          for (int qt = 0; qt < QT; ++qt)
            acc[t][qt] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, kw), q[qt][s], acc[t][qt],
                                                                 0, 0, 0);
        }
      float p[QT][8];
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        float f = a.scale_log2;
        if constexpr (G::W8) f *= ks[e];
#pragma unroll
        for (int qt = 0; qt < QT; ++qt) p[qt][e] = acc[e >> 2][qt][e & 3] * f;
      }
      if (!whole) {
#pragma unroll
        for (int e = 0; e < 8; ++e)
#pragma unroll
          for (int qt = 0; qt < QT; ++qt) p[qt][e] = valid >> e & 1 ? p[qt][e] : -INFINITY;
      }
      st.weigh(p);
      if constexpr (G::W8) {
#pragma unroll
        for (int e = 0; e < 8; ++e)
#pragma unroll
          for (int qt = 0; qt < QT; ++qt) p[qt][e] *= vs[e];
      }
      bf16x8 hi[QT], lo[QT];
      weight_operands<QT, LOW>(p, hi, lo);
      if constexpr (G::W8) {
#pragma unroll
        for (int d = 0; d < G::NW; ++d) {
          uint32_t t[4][2];
          transpose8(r.v, d, t);
#pragma unroll
          for (int j = 0; j < 4; ++j) {
            const u32x2 y = widen4<FMT>(t[j][0]), z = widen4<FMT>(t[j][1]);
            pv_tile<D, QT, LOW>(st, 4 * d + j, __builtin_bit_cast(bf16x8, u32x4{y[0], y[1], z[0], z[1]}), hi, lo);
          }
        }
      } else {
#pragma unroll
        for (int j = 0; j < JT; ++j) pv_tile<D, QT, LOW>(st, j, v_operand16(r.v, j), hi, lo);
      }
    }

    // ---- drafted keys ----
    for (int u = max(u0, en.cached_units); u < u1; ++u) {
      const int key0 = (u - en.cached_units) * kUnit + 32 * w;
      if (!drafts || key0 >= en.cnt) break;
      const uint16_t* kn = static_cast<const uint16_t*>(a.kn.p) + b * a.kn.sb + h * a.kn.sh;
      const uint16_t* vn = static_cast<const uint16_t*>(a.vn.p) + b * a.vn.sb + h * a.vn.sh;
      f32x4 acc[2][QT];
#pragma unroll
      for (int t = 0; t < 2; ++t)
#pragma unroll
        for (int qt = 0; qt < QT; ++qt) acc[t][qt] = f32x4{};
#pragma unroll
      for (int t = 0; t < 2; ++t) {
        const uint16_t* kp = kn + min(key0 + kq + 4 * t + (i16 & 3), en.cnt - 1) * a.kn.sn;
#pragma unroll
        for (int s = 0; s < KS; ++s) {
          bf16x8 kw{};
          const int d = chan<G::W8>(s, g);
          if (d < D) kw = *reinterpret_cast<const bf16x8*>(kp + d);
#pragma unroll
          for (int qt = 0; qt < QT; ++qt)
            acc[t][qt] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(kw, q[qt][s], acc[t][qt], 0, 0, 0);
        }
      }
      uint32_t v[8][JT / 2];
      bool odd = false;                            // a value that is not finite
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        const bool in = key0 + kv8 + e < en.cnt;
        const uint16_t* vp = vn + min(key0 + kv8 + e, en.cnt - 1) * a.vn.sn + min(i16, G::VR - 1) * JT;
#pragma unroll
        for (int d = 0; d < JT / 2; ++d) {
          const uint32_t y = *reinterpret_cast<const uint32_t*>(vp + 2 * d);
          v[e][d] = in ? y : 0u;
          odd |= in && ((y & 0x7F800000u) == 0x7F800000u || (y & 0x7F80u) == 0x7F80u);
        }
      }
      float p[QT][8];
      int seen[QT];
#pragma unroll
      for (int qt = 0; qt < QT; ++qt) {
        const int t = max(tok[qt], 0);
        const uint8_t* mk = a.mask ? a.mask + b * a.mask_b + (int64_t)t * a.T : nullptr;
        seen[qt] = 0;
#pragma unroll
        for (int e = 0; e < 8; ++e) {
          const int key = key0 + kv8 + e;
          const bool on = tok[qt] >= 0 && key < en.cnt && (mk ? mk[min(key, a.T - 1)] != 0 : key <= t);
          seen[qt] |= on ? 1 << e : 0;
          p[qt][e] = on ? acc[e >> 2][qt][e & 3] * a.scale_log2 : -INFINITY;
        }
      }
      st.weigh(p);
      if (__builtin_amdgcn_ballot_w64(odd) != 0) {
        // Inf or NaN among the drafted values (never in practice): 0 * Inf would reach
        // rows that do not see them, so these elements leave the products and are added
        // to the rows that do, one key at a time; weights through LDS, -1 where unseen
        float* pl = &so[w][0][0][0];               // [key][column] of one row tile
#pragma unroll 1
        for (int qt = 0; qt < QT; ++qt) {
#pragma unroll
          for (int e = 0; e < 8; ++e) {
            float y = -1.0f;
#pragma unroll
            for (int c = 0; c < QT; ++c)
              if (c == qt && (seen[c] >> e & 1)) y = p[c][e];
            pl[(kv8 + e) * 16 + i16] = y;
          }
          __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
          const int keys = min(32, en.cnt - key0);
#pragma unroll 1
          for (int key = 0; key < keys; ++key) {
            const float y = pl[key * 16 + i16];
            const bool on = !(y == -1.0f);
#pragma unroll
            for (int r = 0; r < 4; ++r) {
              if (4 * g + r >= G::VR) continue;
              const uint16_t* vp = vn + (key0 + key) * a.vn.sn + JT * (4 * g + r);
#pragma unroll
              for (int j = 0; j < JT; ++j) {
                const float z = __uint_as_float((uint32_t)vp[j] << 16);
                const float add = on && !__builtin_isfinite(z) ? y * z : 0.0f;
#pragma unroll
                for (int c = 0; c < QT; ++c)
                  if (c == qt) st.o[j][c][r] += add;
              }
            }
          }
          __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
        }
#pragma unroll
        for (int e = 0; e < 8; ++e)
#pragma unroll
          for (int d = 0; d < JT / 2; ++d) {
            if ((v[e][d] & 0x7F800000u) == 0x7F800000u) v[e][d] &= 0xFFFFu;
            if ((v[e][d] & 0x7F80u) == 0x7F80u) v[e][d] &= 0xFFFF0000u;
          }
      }
      bf16x8 hi[QT], lo[QT];
      weight_operands<QT, LOW>(p, hi, lo);
#pragma unroll
      for (int j = 0; j < JT; ++j) pv_tile<D, QT, LOW>(st, j, v_operand16(v, j), hi, lo);
    }

    // ---- the four waves meet ----
#pragma unroll
    for (int qt = 0; qt < QT; ++qt) {
      const float l = attn::quad_sum(st.l[qt]);
      if (g == 0) {
        sm[w][qt * 16 + i16] = st.m[qt];
        sl[w][qt * 16 + i16] = l;
      }
    }
    __syncthreads();
    const bool split = u1 - u0 < en.units;
    const int slot = 2 * me + (u0 == 0 ? 1 : 0);
    float* part = a.ws + (int64_t)slot * PT::kFloats;
#pragma unroll
    for (int qt = 0; qt < QT; ++qt) {
      const int row = qt * 16 + i16;
      float top = sm[0][row];
#pragma unroll
      for (int k = 1; k < kWaves; ++k) top = fmaxf(top, sm[k][row]);
      const float ref = top == -INFINITY ? 0.0f : top;
      float l = 0.0f;
#pragma unroll
      for (int k = 0; k < kWaves; ++k) l += sl[k][row] * __builtin_amdgcn_exp2f(sm[k][row] - ref);
      const float mine = __builtin_amdgcn_exp2f(st.m[qt] - ref);
#pragma unroll
      for (int r = 0; r < 4; ++r)
#pragma unroll
        for (int j = 0; j < JT; ++j) so[w][r][lane][j] = st.o[j][qt][r] * mine;
      __syncthreads();
      float y[JT];
#pragma unroll
      for (int j = 0; j < JT; ++j) y[j] = so[0][w][lane][j];
#pragma unroll
      for (int k = 1; k < kWaves; ++k)
#pragma unroll
        for (int j = 0; j < JT; ++j) y[j] += so[k][w][lane][j];
      if (split) {
        float* to = part + ((qt * kWaves + w) * 64 + lane) * JT;
#pragma unroll
        for (int j = 0; j < JT; j += 4) *reinterpret_cast<float4*>(to + j) = make_float4(y[j], y[j + 1], y[j + 2], y[j + 3]);
        if (w == 0 && g == 0) {
          part[PT::kRows * 16 * JT + row] = top;
          part[PT::kRows * 16 * JT + PT::kRows + row] = l;
        }
      } else if (tok[qt] >= 0) {
        const float inv = l == 0.0f ? 0.0f : 1.0f / l;   // NaN stays NaN
        const int d0 = JT * (4 * g + w);
#pragma unroll
        for (int j = 0; j < JT; ++j) y[j] = l == 0.0f ? 0.0f : y[j] * inv;
        if (d0 < D) store_row<D>(a, b, head[qt], tok[qt], d0, y);
        if (a.lse && w == 0 && g == 0)
          a.lse[((int64_t)b * a.H + head[qt]) * a.T + tok[qt]] = l == 0.0f ? -INFINITY : (top + __log2f(l)) * kLn2;
      }
      __syncthreads();
    }
  }
}

// The partial results of one 16-row tile's channels (one of the four that a lane
// row splits into) of a divided segment, joined in the order of the workgroups.
constexpr int kJoinGroups = 4;

template <int D, int QT>
__global__ __launch_bounds__(64 * kJoinGroups) void cache_join_kernel(CacheAttnArgs a, int grid_n, int max_tiles) {
  using PT = Part<D, QT>;
  constexpr int JT = PT::JT, RPT = PT::kRows;
  __shared__ __attribute__((aligned(16))) float so[kJoinGroups][64][JT];
  __shared__ float sm[kJoinGroups][16], sl[kJoinGroups][16];
  const int lane = threadIdx.x & 63, g = lane >> 4, i16 = lane & 15;
  const int grp = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  int id = blockIdx.x;
  const int w = id % kWaves;
  id /= kWaves;
  const int qt = id % QT;
  id /= QT;
  const int rt = id % max_tiles;
  id /= max_tiles;
  const int h = id % a.c.heads, b = id / a.c.heads;

  const Finder fd(a, RPT);
  const Entry en = fd.at(b);
  if (rt >= en.tiles || (rt * RPT + qt * 16) >= en.cnt * a.G) return;
  const int64_t U = fd.total;
  const int n = (int)min((int64_t)grid_n, U);
  // the entry's first unit: the scan up to b
  int64_t base = 0;
  for (int b0 = 0; b0 < b; b0 += 64) {
    const int64_t in = a.B <= 64 ? fd.incl : fd.scan(b0);
    base += __shfl(in, min(b - b0, 64) - 1);
  }
  const int64_t s0 = base + ((int64_t)h * en.tiles + rt) * en.units;
  const int i0 = owner(s0, n, U), i1 = owner(s0 + en.units - 1, n, U);
  if (i0 == i1) return;                            // one workgroup had it all, and wrote it

  auto slot = [&](int i) { return 2 * i + (i == i0 ? 1 : 0); };   // i0's run holds the segment's first unit
  float m = -INFINITY, l = 0.0f;
  float y[JT] = {};
  constexpr int UN = 4;
  for (int k0 = i0 + grp; k0 <= i1; k0 += kJoinGroups * UN) {
    float4 p[UN][JT / 4];
    float pm[UN], pl[UN];
#pragma unroll
    for (int k = 0; k < UN; ++k) {
      const int i = min(k0 + k * kJoinGroups, i1);
      const float* part = a.ws + (int64_t)slot(i) * PT::kFloats;
      const float* from = part + ((qt * kWaves + w) * 64 + lane) * JT;
#pragma unroll
      for (int j = 0; j < JT / 4; ++j) p[k][j] = *reinterpret_cast<const float4*>(from + 4 * j);
      pm[k] = part[RPT * 16 * JT + qt * 16 + i16];
      pl[k] = part[RPT * 16 * JT + RPT + qt * 16 + i16];
    }
#pragma unroll
    for (int k = 0; k < UN; ++k) {
      if (k0 + k * kJoinGroups > i1) break;
      const float to = fmaxf(m, pm[k]);
      const float ref = to == -INFINITY ? 0.0f : to;
      const float f0 = __builtin_amdgcn_exp2f(m - ref), f1 = __builtin_amdgcn_exp2f(pm[k] - ref);
      m = to;
      l = l * f0 + pl[k] * f1;
#pragma unroll
      for (int j = 0; j < JT / 4; ++j) {
        y[4 * j] = y[4 * j] * f0 + p[k][j].x * f1;
        y[4 * j + 1] = y[4 * j + 1] * f0 + p[k][j].y * f1;
        y[4 * j + 2] = y[4 * j + 2] * f0 + p[k][j].z * f1;
        y[4 * j + 3] = y[4 * j + 3] * f0 + p[k][j].w * f1;
      }
    }
  }
#pragma unroll
  for (int j = 0; j < JT; ++j) so[grp][lane][j] = y[j];
  if (g == 0) {
    sm[grp][i16] = m;
    sl[grp][i16] = l;
  }
  __syncthreads();
  if (grp != 0) return;
  float top = sm[0][i16];
#pragma unroll
  for (int k = 1; k < kJoinGroups; ++k) top = fmaxf(top, sm[k][i16]);
  const float ref = top == -INFINITY ? 0.0f : top;
  l = 0.0f;
#pragma unroll
  for (int j = 0; j < JT; ++j) y[j] = 0.0f;
#pragma unroll
  for (int k = 0; k < kJoinGroups; ++k) {
    const float f = __builtin_amdgcn_exp2f(sm[k][i16] - ref);
    l += sl[k][i16] * f;
#pragma unroll
    for (int j = 0; j < JT; ++j) y[j] += so[k][lane][j] * f;
  }
  const int row = rt * RPT + qt * 16 + i16;
  const int t = row / a.G, head = h * a.G + (row - t * a.G);
  if (t >= en.cnt) return;
  const float inv = 1.0f / l;
#pragma unroll
  for (int j = 0; j < JT; ++j) y[j] = l == 0.0f ? 0.0f : y[j] * inv;
  const int d0 = JT * (4 * g + w);
  if (d0 < D) store_row<D>(a, b, head, t, d0, y);
  if (a.lse && w == 0 && g == 0)
    a.lse[((int64_t)b * a.H + head) * a.T + t] = l == 0.0f ? -INFINITY : (top + __log2f(l)) * kLn2;
}

template <int FMT, int D, int QT>
void launch_tile(const CacheAttnArgs& a, const CacheAttnShape& s, hipStream_t stream) {
  if (a.out_f32) hipLaunchKernelGGL((cache_attn_kernel<FMT, D, QT, true>), dim3(s.wgs), dim3(256), 0, stream, a);
  else hipLaunchKernelGGL((cache_attn_kernel<FMT, D, QT, false>), dim3(s.wgs), dim3(256), 0, stream, a);
}

template <int FMT, int D>
void launch_dim(const CacheAttnArgs& a, const CacheAttnShape& s, hipStream_t stream) {
  if (s.qt == 1) launch_tile<FMT, D, 1>(a, s, stream);
  else if (s.qt == 2) launch_tile<FMT, D, 2>(a, s, stream);
  else launch_tile<FMT, D, 4>(a, s, stream);
}

template <int FMT>
hipError_t launch_format(const CacheAttnArgs& a, const CacheAttnShape& s, hipStream_t stream) {
  switch (a.c.D) {
    case 64: launch_dim<FMT, 64>(a, s, stream); break;
    case 112: launch_dim<FMT, 112>(a, s, stream); break;
    case 128: launch_dim<FMT, 128>(a, s, stream); break;
    default: return hipErrorInvalidValue;
  }
  return hipGetLastError();
}

// one translation unit each
hipError_t launch_bf16(const CacheAttnArgs& a, const CacheAttnShape& s, hipStream_t stream);
hipError_t launch_e4m3(const CacheAttnArgs& a, const CacheAttnShape& s, hipStream_t stream);
hipError_t launch_int8(const CacheAttnArgs& a, const CacheAttnShape& s, hipStream_t stream);

}  // namespace cattn
}  // namespace sva
