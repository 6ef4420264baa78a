// Attention of drafted tokens over a paged cache for many query rows per cache head
// (trees; cache_attn_kernel.h has the form for up to 48).
//
// What bounds it: from about 64 rows on a code that is read once meets enough rows
// that widening it, the softmax and the products take longer than reading it (8 ragged
// sequences of up to 75,600 int8 tokens, 6 heads of 128, up to 192 rows: 353 MB and 65 GFLOP in
// 175 us; at full tiles, 8 x 32,768 keys and 128 rows, 103 GFLOP in 155 us, 670 TFLOP/s: vector instructions issue
// in 60% of the cycles, matrix cores are busy in 32%), and
// if every wave widened its own keys, widening would come before the products.  So
// the workgroup's four waves own QT tiles of 16 rows each and share the keys: 64 at
// a time are widened once, by all lanes together, into row-major bf16 tiles in LDS
// (the swizzles and operand reads of attn_w16.h: K by ds_read_b128, V by transpose
// reads), while the raw codes of the next 64 are on their way and the page numbers
// of the 64 after them.  Two stages, one barrier per 64 keys, and no meeting of the
// waves at the end: each has whole rows.
//
// The softmax keeps the running maximum of cache_attn_kernel.h: only where the sum of a
// step's weights exceeds 2^10 (or the row is new) is the step's maximum taken and the
// reference moved, so a weight costs one fma, one exponential and one addition.
#pragma once

#include "cache_attn_common.h"

namespace sva {
namespace cattn {

constexpr int kChunk = 64;       // keys of a stage

// ONE: pages hold whole stages, so that a stage's page and the address of its first row are scalars
// (per row they were a sixth of the vector instructions: 8 ragged sequences of up to 75,600 int8 tokens, up to
// 192 rows, 197 us in pages of 64 without, 187 with)
template <int FMT, int D, int QT, int NP, int AHEAD, bool ONE>
__global__ __launch_bounds__(256) __attribute__((amdgpu_waves_per_eu(2, 2)))
void cache_tile_kernel(CacheAttnArgs a) {
  using G = attn::Geo<D>;
  using G16 = attn::Geo16<D>;
  using PT = Part<D>;
  constexpr bool W8 = FMT != kCacheBf16;
  constexpr int EB = W8 ? 1 : 2;
  constexpr int RPT = 64 * QT, NT = 4 * QT;
  constexpr int LPR = D == 64 ? 4 * EB : 8 * EB;   // lanes of a row, a 16-byte piece each
  constexpr int RPP = 256 / LPR;                   // rows of a pass
  constexpr int NR = kChunk / RPP;                 // rows of a lane
  constexpr int PIECES = D * EB / 16;              // pieces of a row that hold codes
  constexpr int TB = kChunk * G::RB;               // bytes of a tile
  constexpr int NS = QT == 1 ? 2 : 1;              // 32-key steps worked on together
  constexpr int PRE = QT == 1 ? 4 : 2;             // V operands in registers ahead of their use
  __shared__ __attribute__((aligned(1024))) unsigned char Ks[2][TB];
  __shared__ __attribute__((aligned(1024))) unsigned char Vs[2][TB];
  __shared__ __attribute__((aligned(16))) float fs[2][kChunk], vs[2][kChunk];   // K scale * c * log2(e); V scale
  __shared__ __attribute__((aligned(16))) int lost[2][kWaves];   // whether a wave's rows of a stage have a key on a bad page
  __shared__ uint64_t seen[2][RPT];                // which drafted keys of a stage each token of the tile sees
  __shared__ int not_finite;                       // some drafted value of the segment is Inf or NaN

  const int lane = threadIdx.x & 63, g = lane >> 4, i16 = lane & 15;
  // which rows a wave has turns with the workgroup, so that the waves without rows of
  // two workgroups on a CU do not share a SIMD
  const int w = __builtin_amdgcn_readfirstlane(((threadIdx.x >> 6) + blockIdx.x) & 3);
  const int log2p = a.c.log2_page, pmask = (1 << log2p) - 1;
  const int Hkv = a.c.heads;

  const Finder fd(a, RPT, gridDim.x);
  const int64_t W = fd.total;
  if (W == 0) return;
  const int n = (int)min((int64_t)gridDim.x, W);
  const int me = a.G * a.T > RPT && n == (int)gridDim.x ? xcd_remap(blockIdx.x, n) : blockIdx.x;
  if (me >= n) return;
  int64_t x = uniform(run_of(me, n, W));
  const int64_t end = uniform(run_of(me + 1, n, W));
  int64_t ebase;
  int b;

  int koff[G16::KS], voff[G16::DT];
  attn::operand_offsets16<D>(lane, koff, voff);
  const int srow = threadIdx.x / LPR, piece = threadIdx.x % LPR;

  Entry en = fd.locate(x, -1, b, ebase);
  while (x < end) {
    const int64_t work = entry_work(en, Hkv);
    if (x >= ebase + work) {
      ebase += work;
      en = fd.at(++b);
      continue;
    }
    const Piece pc = piece_at(en, x - ebase, end - x);
    const int seg = uniform(pc.seg), u0 = uniform(pc.u0), u1 = uniform(pc.u1);
    x = ebase + uniform(pc.next);
    if (u0 >= u1) continue;
    const int h = uniform(seg / en.tiles), rt = seg - h * en.tiles;

    // ---- Q ----
    bf16x8 q[QT][G16::KS];
    int tok[QT], head[QT];
#pragma unroll
    for (int qt = 0; qt < QT; ++qt) {
      const int row = rt * RPT + (w * QT + qt) * 16 + i16;
      const int t = row / a.G;
      tok[qt] = t < en.cnt ? t : -1;
      head[qt] = h * a.G + (row - t * a.G);
      const uint16_t* p = static_cast<const uint16_t*>(a.q.p) + b * a.q.sb + head[qt] * a.q.sh + t * a.q.sn;
#pragma unroll
      for (int s = 0; s < G16::KS; ++s) {
        const int d = 32 * s + 8 * g;
        if (tok[qt] >= 0 && d < D) q[qt][s] = *reinterpret_cast<const bf16x8*>(p + d);
        else q[qt][s] = bf16x8{};
      }
    }
    // Q has landed here: without this use the compiler waits for it again in every step, and
    // with it for the codes that are on their way
#pragma unroll
    for (int qt = 0; qt < QT; ++qt)
#pragma unroll
      for (int s = 0; s < G16::KS; ++s) asm volatile("" : "+v"(q[qt][s]));
    // a wave without rows stages its share and computes nothing
    const bool busy = rt * RPT + w * QT * 16 < en.cnt * a.G;

    f32x4 o[G16::DT][QT];
    float m[QT], l[QT];
#pragma unroll
    for (int qt = 0; qt < QT; ++qt) {
      m[qt] = -INFINITY;
      l[qt] = 0.0f;
#pragma unroll
      for (int j = 0; j < G16::DT; ++j) o[j][qt] = f32x4{};
    }

    // ---- staging ----
    const int32_t* table = a.table + (int64_t)b * a.max_pages;
    const int k0 = u0 * kUnit;                     // the run's cached keys
    const int k1 = min(en.len, min(u1, en.cached_units) * kUnit);
    const int nc = k1 > k0 ? (k1 - k0 + kChunk - 1) / kChunk : 0;
    auto page_at = [&](int key) { return table[min(key >> log2p, a.max_pages - 1)]; };
    int pg[NR], spg;                               // page numbers of the lane's rows; of its scale's key
    struct Raw {
      u32x4 k[NR], v[NR];
      bool keep[NR];                               // whether the piece is a key's
      bool lost;                                   // a key's page does not exist
      float scale;
      bool scaled;                                 // whether the scale is a key's
    };
    const float* scales = threadIdx.x < kChunk ? a.c.ks : a.c.vs;
    auto load_pages = [&](int c) {
      const int key0 = k0 + c * kChunk;
      if constexpr (ONE) {
        spg = page_at(key0);
        return;
      }
#pragma unroll
      for (int r = 0; r < NR; ++r) pg[r] = page_at(key0 + srow + r * RPP);
      if constexpr (W8) spg = page_at(key0 + (threadIdx.x & (kChunk - 1)));
    };
    // chunk c's codes, with the pages loaded for it, and the next chunk's pages.  Lanes without
    // a key, and all of them past the last chunk, load the cache's first bytes: loads under a
    // condition make the compiler wait for all of them where it needs the older ones only.
    auto load_codes = [&](Raw& x, int c) {
      const int key0 = k0 + c * kChunk;
      int64_t at[NR], sat = 0;
      bool sin = false;
      x.lost = false;
      if constexpr (ONE) {                         // the chunk's page, and its first row: scalars
        const int page = uniform(spg);
        const bool there = page >= 0 && page < a.c.num_pages;
        const int64_t row0 = there ? (((int64_t)page * Hkv + h) << log2p) + (key0 & pmask) : 0;
        x.lost = !there;
        if constexpr (W8) {
          sin = there && key0 + (int)(threadIdx.x & (kChunk - 1)) < k1;
          sat = row0 + (threadIdx.x & (kChunk - 1));
        }
        load_pages(c + 1);
        const uint8_t* kp = static_cast<const uint8_t*>(a.c.k) + row0 * (D * EB);
        const uint8_t* vp = static_cast<const uint8_t*>(a.c.v) + row0 * (D * EB);
        const int off = srow * (D * EB) + min(piece, PIECES - 1) * 16;
#pragma unroll
        for (int r = 0; r < NR; ++r) {
          x.keep[r] = there && key0 + srow + r * RPP < k1 && piece < PIECES;
          x.k[r] = __builtin_nontemporal_load(reinterpret_cast<const u32x4*>(kp + off + r * RPP * D * EB));
          x.v[r] = __builtin_nontemporal_load(reinterpret_cast<const u32x4*>(vp + off + r * RPP * D * EB));
        }
        if constexpr (W8) {
          x.scale = scales[sat];
          x.scaled = sin;
        }
        return;
      }
#pragma unroll
      for (int r = 0; r < NR; ++r) {
        const int key = key0 + srow + r * RPP;
        const bool in = key < k1 && pg[r] >= 0 && pg[r] < a.c.num_pages;
        at[r] = in ? ((((int64_t)pg[r] * Hkv + h) << log2p) + (key & pmask)) * (D * EB) + min(piece, PIECES - 1) * 16 : 0;
        x.keep[r] = in && piece < PIECES;
        x.lost |= key < k1 && !in;
      }
      if constexpr (W8) {
        const int key = key0 + (threadIdx.x & (kChunk - 1));
        sin = key < k1 && spg >= 0 && spg < a.c.num_pages;
        sat = sin ? (((int64_t)spg * Hkv + h) << log2p) + (key & pmask) : 0;
      }
      load_pages(c + 1);                           // (past the end: the table's last column)
#pragma unroll
      for (int r = 0; r < NR; ++r) {
        x.k[r] = __builtin_nontemporal_load(reinterpret_cast<const u32x4*>(static_cast<const uint8_t*>(a.c.k) + at[r]));
        x.v[r] = __builtin_nontemporal_load(reinterpret_cast<const u32x4*>(static_cast<const uint8_t*>(a.c.v) + at[r]));
      }
      if constexpr (W8) {
        x.scale = scales[sat];                     // (the upper half of the lanes loads V's again)
        x.scaled = sin;
      }
    };
    auto write_stage = [&](const Raw& x, int st) {
#pragma unroll
      for (int r = 0; r < NR; ++r) {
        const int row = srow + r * RPP;
        const u32x4 kk = x.keep[r] ? x.k[r] : u32x4{}, vv = x.keep[r] ? x.v[r] : u32x4{};
        if constexpr (W8) {
#pragma unroll
          for (int y = 0; y < 2; ++y) {            // 16 codes make two pieces
            const u32x2 ka = widen4<FMT>(kk[2 * y]), kb = widen4<FMT>(kk[2 * y + 1]);
            const u32x2 va = widen4<FMT>(vv[2 * y]), vb = widen4<FMT>(vv[2 * y + 1]);
            const int c = 2 * piece + y;
            *reinterpret_cast<u32x4*>(&Ks[st][row * G::RB + (attn::swz_k<G::NCH>(row, c) << 4)]) =
                u32x4{ka[0], ka[1], kb[0], kb[1]};
            *reinterpret_cast<u32x4*>(&Vs[st][row * G::RB + (attn::swz_v16<G::NCH>(row, c) << 4)]) =
                u32x4{va[0], va[1], vb[0], vb[1]};
          }
        } else {
          *reinterpret_cast<u32x4*>(&Ks[st][row * G::RB + (attn::swz_k<G::NCH>(row, piece) << 4)]) = kk;
          *reinterpret_cast<u32x4*>(&Vs[st][row * G::RB + (attn::swz_v16<G::NCH>(row, piece) << 4)]) = vv;
        }
      }
      if constexpr (W8) {
        const float y = x.scaled ? x.scale : 0.0f;
        if (threadIdx.x < kChunk) fs[st][threadIdx.x] = y * a.scale_log2;
        else if (threadIdx.x < 2 * kChunk) vs[st][threadIdx.x - kChunk] = y;
      }
      const bool any = __builtin_amdgcn_ballot_w64(x.lost) != 0;
      if (lane == 0) lost[st][threadIdx.x >> 6] = any;
    };

    // a draft chunk, straight from the tensors: values that are not finite are left out
    // (odd: see below)
    const uint16_t* kn = static_cast<const uint16_t*>(a.kn.p) + b * a.kn.sb + h * a.kn.sh;
    const uint16_t* vn = static_cast<const uint16_t*>(a.vn.p) + b * a.vn.sb + h * a.vn.sh;
    const int d0 = max(u0 - en.cached_units, 0) * kUnit;
    const int d1 = a.kn.p ? min(en.cnt, (u1 - en.cached_units) * kUnit) : 0;
    const int nd = d1 > d0 ? (d1 - d0 + kChunk - 1) / kChunk : 0;
    // tokens of the tile's rows; a wave looks at a token's 64 keys at once, eight tokens together
    // (us against each lane's own keys one after the other: 4 sequences of 512 keys and 512 drafted
    // tokens 110 / 86, 64 drafted ones 34 / 31, of one
    // head in place of four 23 / 24; 8 of 8,192 and 60 level)
    const int t0 = rt * RPT / a.G, t1 = min((rt * RPT + RPT - 1) / a.G, en.cnt - 1);
    auto stage_seen = [&](int key0, int st) {
      constexpr int UN = 8;
      const int key = key0 + lane, wv = uniform((int)(threadIdx.x >> 6));
#pragma unroll 1
      for (int t = t0 + wv; t <= t1; t += 4 * UN) {
        int is[UN];
#pragma unroll
        for (int k = 0; k < UN; ++k) {
          const int tk = min(t + 4 * k, t1);
          is[k] = a.mask ? (int)a.mask[b * a.mask_b + (int64_t)tk * a.T + min(key, a.T - 1)] : (int)(key <= tk);
        }
#pragma unroll
        for (int k = 0; k < UN; ++k) {
          const uint64_t bits = __builtin_amdgcn_ballot_w64(is[k] != 0 && key < d1);
          if (lane == 0 && t + 4 * k <= t1) seen[st][t + 4 * k - t0] = bits;
        }
      }
    };
    auto stage_drafts = [&](int key0, int st) {
      bool odd = false;
      stage_seen(key0, st);
#pragma unroll 2
      for (int y = threadIdx.x; y < kChunk * G::NCH; y += 256) {
        const int row = y / G::NCH, c = y % G::NCH, key = key0 + row;
        u32x4 kk{}, vv{};
        if (key < d1 && c < G::DCH) {
          kk = *reinterpret_cast<const u32x4*>(kn + key * a.kn.sn + 8 * c);
          vv = *reinterpret_cast<const u32x4*>(vn + key * a.vn.sn + 8 * c);
        }
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          if ((vv[e] & 0x7F800000u) == 0x7F800000u) { vv[e] &= 0xFFFFu; odd = true; }
          if ((vv[e] & 0x7F80u) == 0x7F80u) { vv[e] &= 0xFFFF0000u; odd = true; }
        }
        *reinterpret_cast<u32x4*>(&Ks[st][row * G::RB + (attn::swz_k<G::NCH>(row, c) << 4)]) = kk;
        *reinterpret_cast<u32x4*>(&Vs[st][row * G::RB + (attn::swz_v16<G::NCH>(row, c) << 4)]) = vv;
      }
      if constexpr (W8) {
        if (threadIdx.x < kChunk) {
          fs[st][threadIdx.x] = a.scale_log2;
          vs[st][threadIdx.x] = 1.0f;
        }
      }
      if (odd) not_finite = 1;
    };
    // the lane's key e of a 32-key step
    auto key_of = [&](int e) { return (e >> 2) * 16 + 4 * g + (e & 3); };
    // which of its eight keys the lane's columns see
    auto seen_cached = [&](int key0, int (&on)[QT]) {
      int bits = 0;
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        const int key = key0 + key_of(e), pp = page_at(key);
        bits |= key < k1 && pp >= 0 && pp < a.c.num_pages ? 1 << e : 0;
      }
#pragma unroll
      for (int qt = 0; qt < QT; ++qt) on[qt] = bits;
    };
    auto seen_drafts = [&](int st, int sub, int (&on)[QT]) {
#pragma unroll
      for (int qt = 0; qt < QT; ++qt) {
        const uint32_t x = tok[qt] >= 0 ? (uint32_t)(seen[st][tok[qt] - t0] >> (32 * sub)) : 0u;
        on[qt] = (int)((x >> 4 * g & 15u) | (x >> (16 + 4 * g) & 15u) << 4);
      }
    };

    // ---- NS 32-key steps from LDS; on: the lane's keys that take part unless whole ----
    auto step = [&](int st, int sub0, bool whole, const int (&on)[NS][QT]) {
      f32x4 s[NS][2][QT];
      const unsigned char* vt = &Vs[st][sub0 * 32 * G::RB];
#pragma unroll
      for (int y = 0; y < NS; ++y) {
        // all K operands are read before the first is used: read where they are used, each
        // was waited for
        const unsigned char* kt = &Ks[st][(sub0 + y) * 32 * G::RB];
        bf16x8 kop[G16::KS][2];
#pragma unroll
        for (int k = 0; k < G16::KS; ++k)
#pragma unroll
          for (int t = 0; t < 2; ++t) kop[k][t] = *reinterpret_cast<const bf16x8*>(kt + koff[k] + t * 16 * G::RB);
        if constexpr (QT > 1) __builtin_amdgcn_sched_barrier(0);
#pragma unroll
        for (int t = 0; t < 2; ++t)
#pragma unroll
          for (int qt = 0; qt < QT; ++qt) s[y][t][qt] = f32x4{};
#pragma unroll
        for (int k = 0; k < G16::KS; ++k)
#pragma unroll
          for (int t = 0; t < 2; ++t)
#pragma unroll
            for (int qt = 0; qt < QT; ++qt)
              s[y][t][qt] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(kop[k][t], q[qt][k], s[y][t][qt], 0, 0, 0);
      }
      // V operands are read ahead of the softmax, as many as registers allow: read where
      // they are used, each pair was waited for
      bf16x8 vop[PRE];
#pragma unroll
      for (int j = 0; j < PRE; ++j) vop[j] = attn::tr_operand16<D>(vt, voff[j]);
      float f[NS][8], z[NS][8];
#pragma unroll
      for (int y = 0; y < NS; ++y)
#pragma unroll
        for (int e = 0; e < 8; e += 4) {
          if constexpr (W8) {
            const int at = (sub0 + y) * 32 + (e >> 2) * 16 + 4 * g;
            const f32x4 u = *reinterpret_cast<const f32x4*>(&fs[st][at]), t = *reinterpret_cast<const f32x4*>(&vs[st][at]);
#pragma unroll
            for (int r = 0; r < 4; ++r) {
              f[y][e + r] = u[r];
              z[y][e + r] = t[r];
            }
          } else {
#pragma unroll
            for (int r = 0; r < 4; ++r) f[y][e + r] = a.scale_log2;
          }
        }
      if (__builtin_expect(!whole, 0)) {
        asm volatile("");                          // a branch that is rarely taken, not selects
#pragma unroll
        for (int y = 0; y < NS; ++y) {
#pragma unroll
          for (int qt = 0; qt < QT; ++qt)
#pragma unroll
            for (int e = 0; e < 8; ++e)
              if (!(on[y][qt] >> e & 1)) s[y][e >> 2][qt][e & 3] = -INFINITY;
          // (an absent key's scale is zero, and 0 * -inf no logit)
          if constexpr (W8) {
#pragma unroll
            for (int e = 0; e < 8; ++e) f[y][e] = f[y][e] == 0.0f && !(on[y][0] >> e & 1) ? 1.0f : f[y][e];
          }
        }
      }
      float p[NS][QT][8], sum[QT];
      auto weigh = [&](int qt, float ref) {
        sum[qt] = 0.0f;
#pragma unroll
        for (int y = 0; y < NS; ++y)
#pragma unroll
          for (int e = 0; e < 8; ++e) {
            p[y][qt][e] = __builtin_amdgcn_exp2f(__builtin_fmaf(s[y][e >> 2][qt][e & 3], f[y][e], -ref));
            sum[qt] += p[y][qt][e];
          }
      };
      // weights are positive: where their sum stays below 2^10, each one does
      bool grow = false;
#pragma unroll
      for (int qt = 0; qt < QT; ++qt) {
        weigh(qt, m[qt]);
        grow |= sum[qt] > 1024.0f || m[qt] == -INFINITY;
      }
      if (__builtin_expect(__builtin_amdgcn_ballot_w64(grow) != 0, 0)) {
        asm volatile("");
#pragma unroll
        for (int qt = 0; qt < QT; ++qt) {
          float top = -INFINITY;
#pragma unroll
          for (int y = 0; y < NS; ++y)
#pragma unroll
            for (int e = 0; e < 8; ++e) top = fmaxf(top, s[y][e >> 2][qt][e & 3] * f[y][e]);
          const float to = fmaxf(m[qt], attn::quad_max(top));
          const float ref = to == -INFINITY ? 0.0f : to;   // only masked keys so far: weights of zero
          const float c = __builtin_amdgcn_exp2f(m[qt] - ref);
          m[qt] = to;
          l[qt] *= c;
#pragma unroll
          for (int j = 0; j < G16::DT; ++j)
#pragma unroll
            for (int r = 0; r < 4; ++r) o[j][qt][r] *= c;
          weigh(qt, ref);
        }
      }
#pragma unroll
      for (int qt = 0; qt < QT; ++qt) l[qt] += sum[qt];
#pragma unroll
      for (int y = 0; y < NS; ++y) {
        if constexpr (W8) {
#pragma unroll
          for (int qt = 0; qt < QT; ++qt)
#pragma unroll
            for (int e = 0; e < 8; ++e) p[y][qt][e] *= z[y][e];
        }
        bf16x8 wp[NP][QT];
        weight_operands<QT, NP>(p[y], wp);
#pragma unroll
        for (int j0 = 0; j0 < G16::DT; j0 += PRE) {
          // the next ones: of this step, or the first of the one after it
          const int jn = j0 + PRE < G16::DT ? j0 + PRE : 0, yn = j0 + PRE < G16::DT ? y : y + 1;
          bf16x8 more[PRE];
#pragma unroll
          for (int j = 0; j < PRE; ++j)
            if (yn < NS && jn + j < G16::DT) more[j] = attn::tr_operand16<D>(vt + yn * 32 * G::RB, voff[jn + j]);
#pragma unroll
          for (int k = 0; k < NP; ++k)
#pragma unroll
            for (int j = 0; j < PRE; ++j)
              if (j0 + j < G16::DT)
#pragma unroll
                for (int qt = 0; qt < QT; ++qt)
                  o[j0 + j][qt] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(vop[j], wp[k][qt], o[j0 + j][qt], 0, 0, 0);
#pragma unroll
          for (int j = 0; j < PRE; ++j) vop[j] = more[j];
        }
      }
    };

    // ---- cached chunks, then drafted ones ----
    if (threadIdx.x == 0) not_finite = 0;
    // AHEAD chunks are on their way beside the one that is worked on
    Raw raw[AHEAD];
    if (nc > 0) {
      load_pages(0);
      load_codes(raw[0], 0);
      if constexpr (AHEAD == 2) load_codes(raw[1], 1);
      write_stage(raw[0], 0);
      load_codes(raw[0], AHEAD);
    } else if (nd > 0) {
      __syncthreads();                             // not_finite is clear
      stage_drafts(d0, 0);
    }
    auto chunk = [&](int c, Raw& next) {           // next: the set with chunk c + 1
      __syncthreads();                             // chunk c is staged; chunk c - 1 is done with
      const int st = c & 1;
      if (c + 1 < nc) {
        write_stage(next, st ^ 1);
        load_codes(next, c + 1 + AHEAD);
      } else if (c + 1 < nc + nd) {
        stage_drafts(d0 + (c + 1 - nc) * kChunk, st ^ 1);
      }
      if (!busy) return;
      const bool cached = c < nc;
      const int key0 = cached ? k0 + c * kChunk : d0 + (c - nc) * kChunk;
      bool whole = false;
      if (cached) whole = key0 + kChunk <= k1 && (lost[st][0] | lost[st][1] | lost[st][2] | lost[st][3]) == 0;
      whole = uniform((int)whole) != 0;
#pragma unroll 1
      for (int sub = 0; sub < 2; sub += NS) {
        int on[NS][QT] = {};
        if (!whole) {
#pragma unroll
          for (int y = 0; y < NS; ++y) {
            if (cached) seen_cached(key0 + 32 * (sub + y), on[y]);
            else seen_drafts(st, sub + y, on[y]);
          }
        }
        step(st, sub, whole, on);
      }
    };
#pragma unroll 1
    for (int c = 0; c < nc + nd; c += AHEAD) {
      chunk(c, raw[AHEAD - 1]);
      if constexpr (AHEAD == 2) {
        if (c + 1 < nc + nd) chunk(c + 1, raw[0]);
      }
    }
    __syncthreads();                               // the stages are free
    // Inf or NaN among the drafted values (never in practice): 0 * Inf would reach rows that
    // do not see them, so they were left out.  For +Inf, -Inf and NaN in turn, a tile of ones
    // where V holds one is multiplied with the rows' masks, and a sum above zero adds that
    // value to the rows that see it.
    if (__builtin_expect(not_finite, 0)) {
#pragma unroll 1
      for (int at = 0; at < 3 * nd; ++at) {
        const int kind = at % 3, key0 = d0 + at / 3 * kChunk;
        stage_seen(key0, 0);
#pragma unroll 1
        for (int y = threadIdx.x; y < kChunk * D; y += 256) {
          const int row = y / D, d = y % D, key = key0 + row;
          const uint16_t bits = key < d1 ? vn[key * a.vn.sn + d] : 0;
          const bool is = kind == 0 ? bits == 0x7F80 : (kind == 1 ? bits == 0xFF80 : (bits & 0x7FFF) > 0x7F80);
          *reinterpret_cast<uint16_t*>(
              &Vs[0][row * G::RB + (attn::swz_v16<G::NCH>(row, d / 8) << 4) + 2 * (d % 8)]) = is ? 0x3F80 : 0;
        }
        __syncthreads();
        const float add = kind == 0 ? INFINITY : (kind == 1 ? -INFINITY : NAN);
#pragma unroll 1
        for (int sub = 0; sub < 2; ++sub) {
          int on[QT];
          seen_drafts(0, sub, on);
          float one[QT][8];
#pragma unroll
          for (int qt = 0; qt < QT; ++qt)
#pragma unroll
            for (int e = 0; e < 8; ++e) one[qt][e] = on[qt] >> e & 1 ? 1.0f : 0.0f;
          bf16x8 wp[1][QT];
          weight_operands<QT, 1>(one, wp);
#pragma unroll
          for (int j = 0; j < G16::DT; ++j) {
            const bf16x8 vop = attn::tr_operand16<D>(&Vs[0][sub * 32 * G::RB], voff[j]);
#pragma unroll
            for (int qt = 0; qt < QT; ++qt) {
              const f32x4 y = __builtin_amdgcn_mfma_f32_16x16x32_bf16(vop, wp[0][qt], f32x4{}, 0, 0, 0);
#pragma unroll
              for (int r = 0; r < 4; ++r) o[j][qt][r] += y[r] > 0.0f ? add : 0.0f;
            }
          }
        }
        __syncthreads();
      }
    }

    // ---- results ----
    const bool split = u1 - u0 < en.units;
    float* part = a.ws + (int64_t)(2 * me + (u0 == 0 ? 1 : 0)) * PT::floats(NT);
#pragma unroll
    for (int qt = 0; qt < QT; ++qt) {
      const float sum = attn::quad_sum(l[qt]);
      const int tile = w * QT + qt;
      if (split) {
#pragma unroll
        for (int j = 0; j < G16::DT; ++j) {
          const int d = 16 * j + 4 * g, cell = d / PT::JT;
          *reinterpret_cast<f32x4*>(part + PT::at(tile, cell & 3, 16 * (cell >> 2) + i16) + d % PT::JT) = o[j][qt];
        }
        if (g == 0) {
          part[PT::ref(NT, tile * 16 + i16)] = m[qt];
          part[PT::sum(NT, tile * 16 + i16)] = sum;
        }
      } else if (tok[qt] >= 0) {
        const float inv = 1.0f / sum;
        const int64_t at = b * a.out.sb + head[qt] * a.out.sh + tok[qt] * a.out.sn + 4 * g;
#pragma unroll
        for (int j = 0; j < G16::DT; ++j) {
          f32x4 y;
#pragma unroll
          for (int r = 0; r < 4; ++r) y[r] = sum == 0.0f ? 0.0f : o[j][qt][r] * inv;
          if (a.out_f32) {
            *reinterpret_cast<f32x4*>(static_cast<float*>(a.out.p) + at + 16 * j) = y;
          } else {
            const u32x2 c = {__builtin_bit_cast(uint32_t, attn::cvt2(y[0], y[1])),
                             __builtin_bit_cast(uint32_t, attn::cvt2(y[2], y[3]))};
            *reinterpret_cast<u32x2*>(static_cast<uint16_t*>(a.out.p) + at + 16 * j) = c;
          }
        }
        if (a.lse && g == 0)
          a.lse[((int64_t)b * a.H + head[qt]) * a.T + tok[qt]] = sum == 0.0f ? -INFINITY : (m[qt] + __log2f(sum)) * kLn2;
      }
    }
  }
}

template <int FMT, int D, int QT>
void launch_tile(const CacheAttnArgs& a, int wgs, hipStream_t stream) {
  constexpr int kAhead = QT == 1 ? 2 : 1;
  auto go = [&](auto kernel) { hipLaunchKernelGGL(kernel, dim3(wgs), dim3(256), 0, stream, a); };
  const bool one = 1 << a.c.log2_page >= kChunk;
  if (a.out_f32 && one) go(cache_tile_kernel<FMT, D, QT, 3, kAhead, true>);
  else if (a.out_f32) go(cache_tile_kernel<FMT, D, QT, 3, kAhead, false>);
  else if (one) go(cache_tile_kernel<FMT, D, QT, 1, kAhead, true>);
  else go(cache_tile_kernel<FMT, D, QT, 1, kAhead, false>);
}

}  // namespace cattn
}  // namespace sva
