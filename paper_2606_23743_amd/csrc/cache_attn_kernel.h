// Attention of drafted tokens over a paged cache: softmax(c Q K^T) V for the
// G * T query rows that share one cache head (row = t * G + g), up to 48 of them
// (cache_attn_tile.h has the form for more).
//
// What bounds it: the keys and values come from HBM once and each code meets at most 48
// rows, so it is bound by HBM, and with few keys by the latency of its chain of
// loads (lengths, pages, K, V).  So the shape is: every wave walks 32-key steps of
// its own with its own running maximum and sum, straight from memory into
// registers (no barrier and no LDS in the loop, whatever the page order; past the caches,
// since nothing is read twice), one step's codes on their way while the step before is
// worked on, and the waves meet once per segment in LDS.  The division of keys among
// workgroups is in cache_attn_plan.h.  48 ragged sequences of up to 32,760 e4m3 tokens, 8 heads of
// 128, four rows each: 841 MB in 142 us, 5.9 TB/s; two of 223,200 in bf16 with 42 rows and
// float32 results: 1,829 MB in 302 us, 6.1 TB/s (a kernel that only reads reaches 6.2, 7.0 past the
// caches); four of up to 1,560: 8.4 us.
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
// The running maximum moves only where a step's weights sum to more than 2^10 (or the row
// is new): weights stay below 2^10 and most steps rescale nothing.
#pragma once

#include "cache_attn_common.h"

namespace sva {
namespace cattn {

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

// one 32-key step as it is in memory
template <int FMT, int D>
struct Raw {
  using G = CGeo<FMT, D>;
  u32x4 k[2][G::NPK];
  uint32_t v[8][G::NW];
  f32x4 ks[2], vs[2];            // 8 bits: scales of the lane's eight keys
  int64_t row;                   // the first of them in the cache
  bool there;                    // their page exists
};

// codes are read once: past the caches
template <class T>
__device__ __forceinline__ T stream(const T* p) { return __builtin_nontemporal_load(p); }

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
template <int D, int QT, int NP>
struct State {
  static constexpr int JT = D > 64 ? 8 : 4;
  f32x4 o[JT][QT];
  float m[QT], l[QT];            // reference (base 2) of the lane's column; the lane's part of the sum
  bf16x8 wp[NP][QT];             // the step's weights as B operands

  __device__ __forceinline__ void clear() {
#pragma unroll
    for (int qt = 0; qt < QT; ++qt) {
      m[qt] = -INFINITY;
      l[qt] = 0.0f;
#pragma unroll
      for (int j = 0; j < JT; ++j) o[j][qt] = f32x4{};
    }
  }

  // logits s * f (base 2; s = -inf where masked) of one row tile -> weights, times z the
  // operands of the product with V.  Weights are positive: where their sum stays below
  // 2^10, each one does, and the reference stays where it is.
  __device__ __forceinline__ void weigh(int qt, const f32x4 (&s)[2], const float (&f)[8], const float (&z)[8], bool scaled) {
    float p[8], sum;
    auto weights = [&](float ref) {
      sum = 0.0f;
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        p[e] = __builtin_amdgcn_exp2f(__builtin_fmaf(s[e >> 2][e & 3], f[e], -ref));
        sum += p[e];
      }
    };
    weights(m[qt]);
    if (__builtin_expect(__builtin_amdgcn_ballot_w64(sum > 1024.0f || m[qt] == -INFINITY) != 0, 0)) {
      asm volatile("");                            // a branch that is rarely taken, not selects
      float top = -INFINITY;
#pragma unroll
      for (int e = 0; e < 8; ++e) top = fmaxf(top, s[e >> 2][e & 3] * f[e]);
      const float to = fmaxf(m[qt], attn::quad_max(top));
      const float ref = to == -INFINITY ? 0.0f : to;   // only masked keys so far: weights of zero
      const float c = __builtin_amdgcn_exp2f(m[qt] - ref);
      m[qt] = to;
      l[qt] *= c;
#pragma unroll
      for (int j = 0; j < JT; ++j)
#pragma unroll
        for (int r = 0; r < 4; ++r) o[j][qt][r] *= c;
      weights(ref);
    }
    l[qt] += sum;
    if (scaled) {
#pragma unroll
      for (int e = 0; e < 8; ++e) p[e] *= z[e];
    }
    float pp[1][8];
    bf16x8 part[NP][1];
#pragma unroll
    for (int e = 0; e < 8; ++e) pp[0][e] = p[e];
    weight_operands<1, NP>(pp, part);
#pragma unroll
    for (int n = 0; n < NP; ++n) wp[n][qt] = part[n][0];
  }

  __device__ __forceinline__ void add(int j, bf16x8 v) {
#pragma unroll
    for (int n = 0; n < NP; ++n)
#pragma unroll
      for (int qt = 0; qt < QT; ++qt)
        o[j][qt] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(v, wp[n][qt], o[j][qt], 0, 0, 0);
  }
};

template <int FMT, int D, int QT, int NP>
__global__ __launch_bounds__(256) __attribute__((amdgpu_waves_per_eu(wave_residents(D, QT))))
void cache_attn_kernel(CacheAttnArgs a) {
  using G = CGeo<FMT, D>;
  using PT = Part<D>;
  constexpr int JT = G::JT, KS = G::KS, RPT = 16 * QT;
  __shared__ __attribute__((aligned(16))) float so[kWaves][4][64][JT];   // one 16-row tile of each wave
  __shared__ __attribute__((aligned(16))) u32x4 qs[QT][KS][64];          // Q as the lanes' B operands
  __shared__ float sm[kWaves][RPT], sl[kWaves][RPT];

  const int lane = threadIdx.x & 63, g = lane >> 4, i16 = lane & 15;
  const int w = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const bool drafts = a.kn.p != nullptr;
  const int log2p = a.c.log2_page, pmask = (1 << log2p) - 1;
  const int Hkv = a.c.heads;

  const Finder fd(a, RPT, gridDim.x);
  const int64_t W = fd.total;
  if (W == 0) return;
  const int n = (int)min((int64_t)gridDim.x, W);
  // neighbouring runs on one XCD where row tiles of a head read the same keys; a grid
  // with workgroups to spare spreads over all XCDs instead
  const int me = a.G * a.T > RPT && n == (int)gridDim.x ? xcd_remap(blockIdx.x, n) : blockIdx.x;
  if (me >= n) return;
  int64_t x = uniform(run_of(me, n, W));
  const int64_t end = uniform(run_of(me + 1, n, W));
  int64_t ebase;                                   // first place of entry b
  int b;

  Entry en = fd.locate(x, -1, b, ebase);
  while (x < end) {
    const int64_t work = entry_work(en, Hkv);
    if (x >= ebase + work) {                       // the next entry
      ebase += work;
      en = fd.at(++b);
      continue;
    }
    const Piece pc = piece_at(en, x - ebase, end - x);
    const int seg = uniform(pc.seg), u0 = uniform(pc.u0), u1 = uniform(pc.u1);
    x = ebase + uniform(pc.next);
    if (u0 >= u1) continue;
    const int h = uniform(seg / en.tiles), rt = seg - h * en.tiles;

    // the token and head of the lane's column in tile qt; token -1: no such row
    auto row_of = [&](int qt, int& tok, int& head) {
      const int row = rt * RPT + qt * 16 + i16, t = row / a.G;
      tok = t < en.cnt ? t : -1;
      head = h * a.G + (row - t * a.G);
    };
    // ---- the first step's pages: nothing waits for Q before its keys are on their way ----
    const int32_t* table = a.table + (int64_t)b * a.max_pages;
    const int kq = 8 * (i16 >> 2), kv8 = 8 * g;    // this lane's K rows and V rows of a step begin here
    auto page_at = [&](int key) { return table[min(key >> log2p, a.max_pages - 1)]; };
    // this wave's steps: units u0 .. ulast - 1 of which its 32 keys begin before the end
    int ulast = min(u1, en.cached_units);
    if (ulast > u0 && (ulast - 1) * kUnit + 32 * w >= en.len) --ulast;
    int pk = 0, pv = 0;
    auto load_pages = [&](int u) {
      pk = page_at(u * kUnit + 32 * w + kq);
      pv = page_at(u * kUnit + 32 * w + kv8);
    };
    if (u0 < ulast) load_pages(u0);

    // ---- Q of this tile's rows ----
    auto load_q = [&](int qt, int s) {
      int t, head;
      row_of(qt, t, head);
      const int d = chan<G::W8>(s, g);
      u32x4 y{};
      if (t >= 0 && d < D)
        y = *reinterpret_cast<const u32x4*>(static_cast<const uint16_t*>(a.q.p) + b * a.q.sb + head * a.q.sh + t * a.q.sn + d);
      return y;
    };
    bf16x8 q1[KS];                                 // one tile stays in registers, more lie in LDS
    if constexpr (QT == 1) {
#pragma unroll
      for (int s = 0; s < KS; ++s) q1[s] = __builtin_bit_cast(bf16x8, load_q(0, s));
    } else {
#pragma unroll 1
      for (int qt = w; qt < QT; qt += kWaves)
#pragma unroll
        for (int s = 0; s < KS; ++s) qs[qt][s][lane] = load_q(qt, s);
      __syncthreads();
    }
    auto q_operand = [&](int qt, int s) {
      if constexpr (QT == 1) return q1[s];
      return __builtin_bit_cast(bf16x8, qs[qt][s][lane]);
    };

    State<D, QT, NP> st;
    st.clear();

    // logits of one row tile: K of 16 keys each in kw[t]
    auto scores = [&](const u32x4 (&kw)[2][KS], int qt, f32x4 (&s)[2]) {
      s[0] = s[1] = f32x4{};
#pragma unroll
      for (int k = 0; k < KS; ++k) {
        const bf16x8 qv = q_operand(qt, k);
#pragma unroll
        for (int t = 0; t < 2; ++t)
          s[t] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, kw[t][k]), qv, s[t], 0, 0, 0);
      }
    };

    // ---- cached keys ----
    // K and its scales, with the pages loaded for it; the next page numbers go out first, so
    // that waiting for them waits for nothing else
    auto load_k = [&](Raw<FMT, D>& r, int u) {
      const int key0 = u * kUnit + 32 * w;
      r.there = pv >= 0 && pv < a.c.num_pages;
      const int64_t gk = pk >= 0 && pk < a.c.num_pages ? pk : 0, gv = r.there ? pv : 0;
      const int64_t rk = ((gk * Hkv + h) << log2p) + ((key0 + kq) & pmask) + (i16 & 3);
      r.row = ((gv * Hkv + h) << log2p) + ((key0 + kv8) & pmask);
      if (u + 1 < ulast) load_pages(u + 1);
      const uint8_t* kp = static_cast<const uint8_t*>(a.c.k) + rk * (D * G::EB);
      // D = 112: groups past the row's end read its last piece, and drop it below
      auto piece = [&](int p) { return min(64 * p + 16 * g, D * G::EB - 16); };
#pragma unroll
      for (int t = 0; t < 2; ++t)
#pragma unroll
        for (int p = 0; p < G::NPK; ++p) r.k[t][p] = stream(reinterpret_cast<const u32x4*>(kp + t * 4 * D * G::EB + piece(p)));
      if constexpr (G::W8) {
#pragma unroll
        for (int e = 0; e < 2; ++e) r.ks[e] = *reinterpret_cast<const f32x4*>(a.c.ks + r.row + 4 * e);
      }
    };
    auto load_v = [&](Raw<FMT, D>& r) {
      if constexpr (G::W8) {
#pragma unroll
        for (int e = 0; e < 2; ++e) r.vs[e] = *reinterpret_cast<const f32x4*>(a.c.vs + r.row + 4 * e);
      }
      const uint8_t* vp = static_cast<const uint8_t*>(a.c.v) + r.row * (D * G::EB) + min(i16, G::VR - 1) * JT * G::EB;
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        const uint8_t* p = vp + e * D * G::EB;
        if constexpr (G::NW == 1) {
          r.v[e][0] = stream(reinterpret_cast<const uint32_t*>(p));
        } else if constexpr (G::NW == 2) {
          const u32x2 y = stream(reinterpret_cast<const u32x2*>(p));
          r.v[e][0] = y[0];
          r.v[e][1] = y[1];
        } else {
          const u32x4 y = stream(reinterpret_cast<const u32x4*>(p));
          r.v[e][0] = y[0];
          r.v[e][1] = y[1];
          r.v[e][2] = y[2];
          r.v[e][3] = y[3];
        }
      }
    };
    // One step.  K of the next one is loaded as soon as this one's is widened (bf16:
    // multiplied) and V as soon as it is transposed: into the registers that this frees, so
    // that a step's codes are on their way while the step before is worked on.  (Two sets in
    // turn took 32 to 64 registers more; at D = 128 they were no faster in 8 bits, 137 us both for
    // 840 MB, and spilled in bf16, 450 us for 279.)
    auto work_on = [&](Raw<FMT, D>& r, int u) {
      const int left = en.len - u * kUnit - 32 * w;
      const bool there = r.there, whole = left >= 32 && __builtin_amdgcn_ballot_w64(!there) == 0;
      float f[8], z[8];
#pragma unroll
      for (int e = 0; e < 8; ++e) f[e] = G::W8 ? a.scale_log2 * r.ks[e >> 2][e & 3] : a.scale_log2;
      u32x4 kw[2][KS];
#pragma unroll
      for (int s = 0; s < KS; ++s)
#pragma unroll
        for (int t = 0; t < 2; ++t) {
          if constexpr (G::W8) {
            const u32x2 y = widen4<FMT>(r.k[t][s >> 1][2 * (s & 1)]), c = widen4<FMT>(r.k[t][s >> 1][2 * (s & 1) + 1]);
            kw[t][s] = u32x4{y[0], y[1], c[0], c[1]};
          } else {
            kw[t][s] = r.k[t][s];
          }
          if (D == 112 && chan<G::W8>(s, 3) >= D) {  // a step with absent channels
            if (chan<G::W8>(s, g) >= D) kw[t][s] = u32x4{};
          }
        }
      if constexpr (G::W8) {
        if (u + 1 < ulast) load_k(r, u + 1);
      }
      int on = 0xff;
      if (__builtin_expect(!whole, 0)) {           // the sequence's last keys, or a bad page
        asm volatile("");
#pragma unroll
        for (int e = 0; e < 8; ++e)
          if (!there || kv8 + e >= left) {
            on &= ~(1 << e);
            f[e] = 1.0f;
            if constexpr (G::W8) r.vs[e >> 2][e & 3] = 0.0f;
#pragma unroll
            for (int d = 0; d < G::NW; ++d) r.v[e][d] = 0;
          }
      }
#pragma unroll
      for (int e = 0; e < 8; ++e) z[e] = G::W8 ? r.vs[e >> 2][e & 3] : 1.0f;
#pragma unroll
      for (int qt = 0; qt < QT; ++qt) {
        if constexpr (QT > 1) __builtin_amdgcn_sched_barrier(0);   // one tile's logits at a time
        f32x4 s[2];
        scores(kw, qt, s);
        if (__builtin_expect(!whole, 0)) {
          asm volatile("");
#pragma unroll
          for (int e = 0; e < 8; ++e)
            if (!(on >> e & 1)) s[e >> 2][e & 3] = -INFINITY;
        }
        st.weigh(qt, s, f, z, G::W8);
      }
      if constexpr (!G::W8) {
        if (u + 1 < ulast) load_k(r, u + 1);
      }
      if constexpr (G::W8) {
#pragma unroll
        for (int d = 0; d < G::NW; ++d) {
          __builtin_amdgcn_sched_barrier(0);
          uint32_t t[4][2];
          transpose8(r.v, d, t);
#pragma unroll
          for (int j = 0; j < 4; ++j) {
            const u32x2 y = widen4<FMT>(t[j][0]), c = widen4<FMT>(t[j][1]);
            st.add(4 * d + j, __builtin_bit_cast(bf16x8, u32x4{y[0], y[1], c[0], c[1]}));
          }
        }
      } else {
#pragma unroll
        for (int j = 0; j < JT; ++j) {
          if (j % 2 == 0) __builtin_amdgcn_sched_barrier(0);
          st.add(j, v_operand16(r.v, j));
        }
      }
      if (u + 1 < ulast) load_v(r);
    };
    if (u0 < ulast) {
      Raw<FMT, D> r;
      load_k(r, u0);
      load_v(r);
      // Q has landed here: without this use the compiler waits for it again in every step,
      // and with it for the codes that are on their way
      if constexpr (QT == 1) {
#pragma unroll
        for (int s = 0; s < KS; ++s) asm volatile("" : "+v"(q1[s]));
      }
      for (int u = u0; u < ulast; ++u) work_on(r, u);
    }

    // ---- drafted keys ----
    const uint16_t* kn = static_cast<const uint16_t*>(a.kn.p) + b * a.kn.sb + h * a.kn.sh;
    const uint16_t* vn = static_cast<const uint16_t*>(a.vn.p) + b * a.vn.sb + h * a.vn.sh;
    // which of its eight keys the lane's column sees
    auto seen_drafts = [&](int qt, int key0) {
      int t, head;
      row_of(qt, t, head);
      const uint8_t* mk = a.mask ? a.mask + b * a.mask_b + (int64_t)max(t, 0) * a.T : nullptr;
      int seen = 0;
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        const int key = key0 + kv8 + e;
        seen |= t >= 0 && key < en.cnt && (mk ? mk[min(key, a.T - 1)] != 0 : key <= t) ? 1 << e : 0;
      }
      return seen;
    };
    // a drafted value row's channels of this lane; zero behind the last token
    auto load_vn = [&](int key, uint32_t (&v)[JT / 2]) {
      const uint16_t* vp = vn + min(key, en.cnt - 1) * a.vn.sn + min(i16, G::VR - 1) * JT;
#pragma unroll
      for (int d = 0; d < JT / 2; ++d) {
        const uint32_t y = *reinterpret_cast<const uint32_t*>(vp + 2 * d);
        v[d] = key < en.cnt ? y : 0u;
      }
    };
    bool not_finite = false;
#pragma unroll 1
    for (int u = max(u0, en.cached_units); u < u1; ++u) {
      const int key0 = (u - en.cached_units) * kUnit + 32 * w;
      if (!drafts || key0 >= en.cnt) break;
      u32x4 kw[2][KS];
#pragma unroll
      for (int t = 0; t < 2; ++t) {
        const uint16_t* kp = kn + min(key0 + kq + 4 * t + (i16 & 3), en.cnt - 1) * a.kn.sn;
#pragma unroll
        for (int s = 0; s < KS; ++s) {
          const int d = chan<G::W8>(s, g);
          kw[t][s] = *reinterpret_cast<const u32x4*>(kp + min(d, D - 8));
          if (D == 112 && d >= D) kw[t][s] = u32x4{};
        }
      }
      uint32_t v[8][JT / 2];
      bool odd = false;                            // a value that is not finite
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        load_vn(key0 + kv8 + e, v[e]);
#pragma unroll
        for (int d = 0; d < JT / 2; ++d)
          odd |= (v[e][d] & 0x7F800000u) == 0x7F800000u || (v[e][d] & 0x7F80u) == 0x7F80u;
      }
      const float f[8] = {a.scale_log2, a.scale_log2, a.scale_log2, a.scale_log2,
                          a.scale_log2, a.scale_log2, a.scale_log2, a.scale_log2};
#pragma unroll
      for (int qt = 0; qt < QT; ++qt) {
        f32x4 s[2];
        scores(kw, qt, s);
        const int seen = seen_drafts(qt, key0);
#pragma unroll
        for (int e = 0; e < 8; ++e)
          if (!(seen >> e & 1)) s[e >> 2][e & 3] = -INFINITY;
        st.weigh(qt, s, f, f, false);
      }
      if (__builtin_expect(__builtin_amdgcn_ballot_w64(odd) != 0, 0)) {
        not_finite = true;                         // 0 * Inf would reach rows that do not see it: added below
#pragma unroll
        for (int e = 0; e < 8; ++e)
#pragma unroll
          for (int d = 0; d < JT / 2; ++d) {
            if ((v[e][d] & 0x7F800000u) == 0x7F800000u) v[e][d] &= 0xFFFFu;
            if ((v[e][d] & 0x7F80u) == 0x7F80u) v[e][d] &= 0xFFFF0000u;
          }
      }
#pragma unroll
      for (int j = 0; j < JT; ++j) st.add(j, v_operand16(v, j));
    }
    // Inf or NaN among the drafted values (never in practice) were left out of the products.
    // For +Inf, -Inf and NaN in turn, a matrix of ones where V holds one is multiplied with
    // the rows' masks, and a sum above zero adds that value to the rows that see it.
    if (__builtin_expect(not_finite, 0)) {
#pragma unroll 1
      for (int u = max(u0, en.cached_units); u < u1; ++u) {
        const int key0 = (u - en.cached_units) * kUnit + 32 * w;
        if (key0 >= en.cnt) break;
        uint32_t v[8][JT / 2];
#pragma unroll
        for (int e = 0; e < 8; ++e) load_vn(key0 + kv8 + e, v[e]);
        bf16x8 mask_op[QT];
#pragma unroll
        for (int qt = 0; qt < QT; ++qt) {
          const int seen = seen_drafts(qt, key0);
          float one[1][8];
          bf16x8 part[1][1];
#pragma unroll
          for (int e = 0; e < 8; ++e) one[0][e] = seen >> e & 1 ? 1.0f : 0.0f;
          weight_operands<1, 1>(one, part);
          mask_op[qt] = part[0][0];
        }
#pragma unroll 1
        for (int kind = 0; kind < 3; ++kind) {
          const float add = kind == 0 ? INFINITY : (kind == 1 ? -INFINITY : NAN);
          // bits & care within span of the first: +Inf; -Inf; NaN of either sign
          const uint32_t care = kind == 2 ? 0x7FFFu : 0xFFFFu, from = kind == 0 ? 0x7F80u : (kind == 1 ? 0xFF80u : 0x7F81u);
          const uint32_t span = kind == 2 ? 0x7Eu : 0u;
#pragma unroll
          for (int e = 0; e < 8; ++e)
#pragma unroll
            for (int d = 0; d < JT / 2; ++d) asm volatile("" : "+v"(v[e][d]));   // (no marks made ahead of the loop)
#pragma unroll
          for (int j = 0; j < JT; ++j) {
            __builtin_amdgcn_sched_barrier(0);     // one tile at a time: its marks need not live longer
            uint32_t t[8][1];
#pragma unroll
            for (int e = 0; e < 8; ++e)
              t[e][0] = ((j & 1 ? v[e][j >> 1] >> 16 : v[e][j >> 1] & 0xFFFFu) & care) - from <= span ? 0x3F80u : 0u;
            const bf16x8 marks = v_operand16(t, 0);
#pragma unroll
            for (int qt = 0; qt < QT; ++qt) {
              const f32x4 y = __builtin_amdgcn_mfma_f32_16x16x32_bf16(marks, mask_op[qt], f32x4{}, 0, 0, 0);
#pragma unroll
              for (int r = 0; r < 4; ++r) st.o[j][qt][r] += y[r] > 0.0f ? add : 0.0f;
            }
          }
        }
      }
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
    float* part = a.ws + (int64_t)slot * PT::floats(QT);
#pragma unroll
    for (int qt = 0; qt < QT; ++qt) {
      const int row = qt * 16 + i16;
      int tok, head;
      row_of(qt, tok, head);
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
        float* to = part + PT::at(qt, w, lane);
#pragma unroll
        for (int j = 0; j < JT; j += 4) *reinterpret_cast<float4*>(to + j) = make_float4(y[j], y[j + 1], y[j + 2], y[j + 3]);
        if (w == 0 && g == 0) {
          part[PT::ref(QT, row)] = top;
          part[PT::sum(QT, row)] = l;
        }
      } else if (tok >= 0) {
        const float inv = l == 0.0f ? 0.0f : 1.0f / l;   // NaN stays NaN
        const int d0 = JT * (4 * g + w);
#pragma unroll
        for (int j = 0; j < JT; ++j) y[j] = l == 0.0f ? 0.0f : y[j] * inv;
        if (d0 < D) store_row<D>(a, b, head, tok, d0, y);
        if (a.lse && w == 0 && g == 0)
          a.lse[((int64_t)b * a.H + head) * a.T + tok] = l == 0.0f ? -INFINITY : (top + __log2f(l)) * kLn2;
      }
      __syncthreads();
    }
  }
}

template <int FMT, int D, int QT>
void launch_wave(const CacheAttnArgs& a, int wgs, hipStream_t stream) {
  if (a.out_f32) hipLaunchKernelGGL((cache_attn_kernel<FMT, D, QT, 3>), dim3(wgs), dim3(256), 0, stream, a);
  else hipLaunchKernelGGL((cache_attn_kernel<FMT, D, QT, 1>), dim3(wgs), dim3(256), 0, stream, a);
}

}  // namespace cattn
}  // namespace sva
