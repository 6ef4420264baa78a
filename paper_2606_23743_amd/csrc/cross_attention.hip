// Cross attention: softmax(c Q K^T) V of N query tokens over the M states of an
// encoder, heads in groups that share keys, keys hidden by a length or a mask.
//
// A workgroup holds 128 (64) rows of one kv head, a row being a token of one of the
// group's heads, so keys are read once for the whole group and a single token's heads
// fill a tile; its four waves take 32 (16) rows each.  Keys go by in tiles of 32 that
// every wave reads from LDS, filled three tiles ahead by direct loads; the wave's
// arithmetic is that of attn_w16.h, S of the next tile beside the softmax of this one.
// The reference of a row's weights is a running maximum that moves only when a logit
// passes it by 2^30, so weights, their sum and O stay far inside float32 while O is
// almost never rescaled.  O is divided by the sum of the weights as they were rounded
// to bf16 for the product, the log-sum-exp is that of the unrounded ones.
// A length ends the walk, as a mask's last seen key does; keys that a mask hides before it
// are loaded as zeros and their logits replaced.  Where few rows meet many keys, the keys
// are divided among workgroups and their results joined by a second launch.
//
// Bound by the step's chain of S, softmax and product at the clock the power limit leaves,
// and by the rows' traffic, which with few keys comes on top of it: 63,240 rows of 32 heads
// of 128 over 512 keys 680 us (780 TFLOP/s; 1.04 GB), 16,384 rows of 4 heads over as many keys
// 540 us (1,020 TFLOP/s), 32,760 rows of 2 x 20 heads of 112 over 512 keys 450 us, with a
// tenth of them hidden by holes in a mask 510.  Few rows are bound by HBM: 2 x 7 tokens of 48
// heads over 111,600 keys 173 us (5.3 TB/s).
#include "cross_tiles.h"

namespace sva {
namespace {

using namespace cross;

constexpr int NST = 4, PD = 3;   // LDS stages, tiles ahead

// a row's reference moves when a logit passes it by this much (log2 units)
constexpr float kSlack = 30.0f;

// What a wave keeps of its rows: the weights' reference (log2 units), their sums as rounded
// to bf16 and unrounded (this lane's quarter), and O^T before it is divided.
template <int D, int QT, bool LSE>
struct RowState {
  static constexpr int DT = Geo16<D>::DT;
  float m_ref[QT], limit[QT], l_part[QT], l_full[QT];
  f32x4 oacc[DT][QT];

  __device__ __forceinline__ void clear() {
#pragma unroll
    for (int qt = 0; qt < QT; ++qt) {
      m_ref[qt] = -3e38f;
      limit[qt] = -INFINITY;
      l_part[qt] = l_full[qt] = 0.0f;
#pragma unroll
      for (int dt = 0; dt < DT; ++dt) oacc[dt][qt] = f32x4{};
    }
  }
  // moves the reference of rows that have a logit above their limit
  __device__ __forceinline__ void follow(const f32x4 (&s)[2][QT], float sl2) {
    float mx[QT];
    bool over = false;
#pragma unroll
    for (int qt = 0; qt < QT; ++qt) {
      mx[qt] = s[0][qt][0];
#pragma unroll
      for (int k2 = 0; k2 < 2; ++k2)
#pragma unroll
        for (int r = 0; r < 4; ++r) mx[qt] = fmaxf(mx[qt], s[k2][qt][r]);
      over |= mx[qt] > limit[qt];
    }
    if (__builtin_amdgcn_ballot_w64(over) != 0) {
      asm volatile("");
#pragma unroll
      for (int qt = 0; qt < QT; ++qt) {
        const float m_new = fmaxf(m_ref[qt], quad_max(mx[qt]) * sl2);
        const float f = __builtin_amdgcn_exp2f(m_ref[qt] - m_new);
        l_part[qt] *= f;
        if constexpr (LSE) l_full[qt] *= f;
#pragma unroll
        for (int dt = 0; dt < DT; ++dt)
#pragma unroll
          for (int r = 0; r < 4; ++r) oacc[dt][qt][r] *= f;
        m_ref[qt] = m_new;
        limit[qt] = (m_new + kSlack) / sl2;
      }
    }
  }
  __device__ __forceinline__ void weigh(const f32x4 (&s)[2][QT], bf16x8 (&pop)[QT], float sl2) {
    const bf16x2 ones = {(__bf16)1.0f, (__bf16)1.0f};
#pragma unroll
    for (int qt = 0; qt < QT; ++qt) {
      u32x4 wv;
      float lsum = l_part[qt], lf = l_full[qt];
#pragma unroll
      for (int k2 = 0; k2 < 2; ++k2)
#pragma unroll
        for (int e = 0; e < 2; ++e) {
          const float p0 = __builtin_amdgcn_exp2f(__builtin_fmaf(s[k2][qt][2 * e], sl2, -m_ref[qt]));
          const float p1 = __builtin_amdgcn_exp2f(__builtin_fmaf(s[k2][qt][2 * e + 1], sl2, -m_ref[qt]));
          const bf16x2 pb = cvt2(p0, p1);
          lsum = __builtin_amdgcn_fdot2_f32_bf16(pb, ones, lsum, false);
          if constexpr (LSE) lf += p0 + p1;
          wv[k2 * 2 + e] = __builtin_bit_cast(unsigned, pb);
        }
      pop[qt] = __builtin_bit_cast(bf16x8, wv);
      l_part[qt] = lsum;
      if constexpr (LSE) l_full[qt] = lf;
    }
  }
};

template <int D, int QT, bool MASK, bool LSE>
__global__ __launch_bounds__(kThreads) __attribute__((amdgpu_waves_per_eu(wide_per_cu(D), QT == 2 ? wide_per_cu(D) : 4)))
void cross_attn_kernel(CrossArgs a) {
  using G16 = Geo16<D>;
  using Feed = KeyFeed<D, MASK, false>;
  constexpr int CT = TileLoader<D>::CT;
  __shared__ __attribute__((aligned(1024))) unsigned char Ks[NST][CT];
  __shared__ __attribute__((aligned(1024))) unsigned char Vs[NST][CT];

  const int lane = threadIdx.x & 63, i = lane & 15, g = lane >> 4;
  const int w = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const float sl2 = a.scale_log2;
  const unsigned ks_base = __builtin_amdgcn_readfirstlane((unsigned)(size_t)(const lds_u8*)&Ks[0][0]);
  const unsigned vs_base = __builtin_amdgcn_readfirstlane((unsigned)(size_t)(const lds_u8*)&Vs[0][0]);

  const Item it(a);
  const int64_t bh = (int64_t)it.b * a.Hkv + it.kvh;
  auto row_of = [&](int tile, int qt) { return tile * 64 * QT + (w * QT + qt) * 16 + i; };
  auto load_q = [&](bf16x8 (&op)[QT][G16::KS], int tile) {
    const uint16_t* rows[QT];
#pragma unroll
    for (int qt = 0; qt < QT; ++qt) {
      const int r = row_of(tile, qt);
      rows[qt] = r < a.R ? static_cast<const uint16_t*>(a.q.p) + row_offset(a.q, it.b, it.kvh * a.G, r, a.N, a.G) : nullptr;
    }
    load_operand<D>(op, rows, lane);
  };

  int koff[G16::KS], voff[G16::DT];
  operand_offsets<D>(lane, koff, voff);
  RowState<D, QT, LSE> rs;
  auto store = [&](int tile) {
#pragma unroll
    for (int qt = 0; qt < QT; ++qt) {
      const float l_tot = quad_sum(rs.l_part[qt]);
      const float l_all = LSE ? quad_sum(rs.l_full[qt]) : l_tot;
      const int r = row_of(tile, qt);
      const bool there = r < a.R;
      if (a.splits > 1) {
        if (!there) continue;
        const int64_t at = (bh * a.splits + it.split) * a.R + r;
        float* o = a.part + at * D;
#pragma unroll
        for (int dt = 0; dt < G16::DT; ++dt) *reinterpret_cast<f32x4*>(o + dt * 16 + 4 * g) = rs.oacc[dt][qt];
        if (g == 0) {
          a.stat[at] = make_float2(rs.m_ref[qt], l_tot);
          if constexpr (LSE) a.stat_l[at] = l_all;
        }
        continue;
      }
      const bool has = l_tot > 0.0f || l_tot != l_tot;   // a NaN stays one
      uint16_t* o = there ? static_cast<uint16_t*>(a.out.p) + row_offset(a.out, it.b, it.kvh * a.G, r, a.N, a.G) : nullptr;
      store_row<D>(o, &rs.oacc[0][qt], QT, has ? 1.0f / l_tot : 0.0f, g);
      if constexpr (LSE) {
        if (g == 0 && there) a.lse[bh * a.R + r] = has ? (rs.m_ref[qt] + __log2f(l_all)) * 0.69314718055994530942f : -INFINITY;
      }
    }
  };

  rs.clear();
  if (it.chunks == 0) {            // no key: zeros
    for (int t = 0; t < it.tiles; ++t) store(it.tile + t);
    return;
  }
  Feed feed;
  feed.start(a, it, w, lane);
  feed.ld.clear_pads(&Ks[0][0], NST);
  feed.ld.clear_pads(&Vs[0][0], NST);
  auto fetch = [&](int st) { return feed.feed(a, ks_base + st * CT, vs_base + st * CT); };
  bf16x8 qop[QT][G16::KS], qnext[QT][G16::KS];
  load_q(qop, it.tile);
  // keys seen of the tiles ahead
  uint32_t seen[PD];
#pragma unroll
  for (int c = 0; c < PD; ++c) seen[c] = fetch(c);
  wait_vmcnt_lds_idle<Feed::kLoads * (PD - 1)>();      // tile 0 has landed, Q before it
  wg_barrier();
  f32x4 sacc[2][QT];
  qk16<D>(sacc, &Ks[0][0], koff, qop);
  if (seen[0] != ~0u) {
    settle(sacc[0], sacc[1]);
    hide(sacc, seen[0], lane);
  }

  // A step is one tile of keys, in stage st: its softmax and product with V, and S of the
  // tile after it, which past the last is the first one again for the next row tile.
  int st = 0, c = 0, late = 0, tile = it.tile;
  const int end = it.tile + it.tiles, ahead = max(it.chunks - 4, 0);
  bool pending = false;            // a row tile whose result is not stored yet
#pragma unroll 1
  while (true) {
    // The next tile has landed; in the two steps after Q's loads those may still be under way.
    if (late > 0) wait_vmcnt_lds_idle<Feed::kLoads * (PD - 2) + QT * G16::KS>();
    else wait_vmcnt_lds_idle<Feed::kLoads * (PD - 2)>();
    --late;
    wg_barrier();                  // and every wave is done with the tile before
    if (pending) {                 // (stored here, ahead of loads that are waited for two steps later)
      store(tile - 1);
      rs.clear();
      pending = false;
      if (tile == end) break;
    }
    const uint32_t fed = fetch((st + PD) % NST);
    if (c == ahead) {              // Q of the next row tile, four tiles of keys before it is used
      asm volatile("" ::: "memory");     // behind the tile's loads: the next waits count on it
      if (tile + 1 < end) {
        load_q(qnext, tile + 1);
        late = 2;
      }
    }
    rs.follow(sacc, sl2);
    if (++c == it.chunks) {
      c = 0;
      ++tile;
      pending = true;
#pragma unroll
      for (int qt = 0; qt < QT; ++qt)
#pragma unroll
        for (int s = 0; s < G16::KS; ++s) qop[qt][s] = qnext[qt][s];
    }
    f32x4 snext[2][QT];
    bf16x8 pop[QT];
    qk16<D>(snext, &Ks[0][0] + (st + 1) % NST * CT, koff, qop);
    rs.weigh(sacc, pop, sl2);
    __builtin_amdgcn_s_setprio(1);
    pv16<D>(pop, &Vs[0][0] + st * CT, voff, rs.oacc);
    __builtin_amdgcn_s_setprio(0);
    if (__builtin_expect(seen[1] != ~0u, 0)) {
      asm volatile("");
      hide(snext, seen[1], lane);
    }
#pragma unroll
    for (int x = 1; x < PD; ++x) seen[x - 1] = seen[x];
    seen[PD - 1] = fed;
#pragma unroll
    for (int x = 0; x < 2; ++x)
#pragma unroll
      for (int qt = 0; qt < QT; ++qt) sacc[x][qt] = snext[x][qt];
    st = (st + 1) % NST;
  }
  wait_vmcnt<0>();                 // no load may still target this workgroup's LDS
}

// Sixteen rows at most (a single token's heads): the keys are the work, and a chain of
// steps the time.  So the four waves of a workgroup take a tile of keys each, with stages of
// their own and no barrier between them, and join their states at the end.  31 x 32 heads
// of one token over 4,000 keys of 64 take 167 us (6.1 TB/s) instead of 243 with the kernel
// above, 8 x 32 heads over 8 x 1,560 keys of 128 13.4 instead of 14.6, over 512 keys of one
// entry 6.7 instead of 9.4.
template <int D, bool MASK, bool LSE>
__global__ __launch_bounds__(kThreads) void cross_few_kernel(CrossArgs a) {
  using G = Geo<D>;
  using G16 = Geo16<D>;
  constexpr int CT = TileLoader<D>::CT, NU = CT / 1024, kStages = 2, kWaves = kThreads / 64;
  // stages of K and V for each wave; then the waves' O, 16 rows of D
  __shared__ __attribute__((aligned(1024))) unsigned char Ts[kWaves][kStages][2][CT];
  __shared__ float ms[kWaves][16], ls[kWaves][16], lf[kWaves][16];
  static_assert(kStages * 2 * CT >= 16 * D * 4, "a wave's O fits its stages");

  const int lane = threadIdx.x & 63, i = lane & 15, g = lane >> 4;
  const int w = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const float sl2 = a.scale_log2;
  const Item it(a);
  const int64_t bh = (int64_t)it.b * a.Hkv + it.kvh;
  unsigned char* mine = &Ts[w][0][0][0];
  const unsigned base = __builtin_amdgcn_readfirstlane((unsigned)(size_t)(const lds_u8*)mine);

  const uint16_t* rows[1] = {
      i < a.R ? static_cast<const uint16_t*>(a.q.p) + row_offset(a.q, it.b, it.kvh * a.G, i, a.N, a.G) : nullptr};
  bf16x8 qop[1][G16::KS];
  load_operand<D>(qop, rows, lane);
  RowState<D, 1, LSE> rs;
  rs.clear();

  // this wave's tiles: it.c0 + w, + kWaves, ...
  const uint32_t* words = MASK ? a.bits + (int64_t)it.b * ((a.M + 31) / 32) : nullptr;
  const int last = it.c0 + it.chunks;
  auto seen_of = [&](int c) -> uint32_t {
    if (c >= last) return 0u;
    if constexpr (MASK) return *(const __attribute__((address_space(4))) uint32_t*)(words + c);
    return rows_left(it.count - c * CK);
  };
  const uint16_t* Kh = static_cast<const uint16_t*>(a.k.p) + it.b * a.k.sb + it.kvh * a.k.sh;
  const uint16_t* Vh = static_cast<const uint16_t*>(a.v.p) + it.b * a.v.sb + it.kvh * a.v.sh;
  // all of a tile's pieces, zeros where a row is not seen or a piece not there
  auto fetch = [&](int st, int c, uint32_t seen) {
#pragma unroll
    for (int t = 0; t < 2; ++t) {
      const int64_t pitch = t ? a.v.sn : a.k.sn;
      const uint16_t* tile = (t ? Vh : Kh) + (int64_t)c * CK * pitch;
#pragma unroll
      for (int u = 0; u < NU; ++u) {
        const int r = u * G::RPI + lane / G::NCH, p = swz<G::NCH>(r, lane % G::NCH);
        const void* from = tile + r * pitch + p * 8;
        global_to_lds<16>((seen >> r & 1) && p < G::DCH ? from : (const void*)kZeros, base + (st * 2 + t) * CT + u * 1024);
      }
    }
  };
  int koff[G16::KS], voff[G16::DT];
  operand_offsets<D>(lane, koff, voff);
  uint32_t seen[kStages];
#pragma unroll
  for (int st = 0; st < kStages; ++st) {
    seen[st] = seen_of(it.c0 + w + st * kWaves);
    fetch(st, it.c0 + w + st * kWaves, seen[st]);
  }
  int st = 0;
#pragma unroll 1
  for (int c = it.c0 + w; c < last; c += kWaves) {
    wait_vmcnt<2 * NU*(kStages - 1)>();          // the tile has landed
    const unsigned char* kt = mine + st * 2 * CT;
    f32x4 s[2][1];
    qk16<D>(s, kt, koff, qop);
    settle(s[0], s[1]);
    if (seen[0] != ~0u) hide(s, seen[0], lane);
    rs.follow(s, sl2);
    bf16x8 pop[1];
    rs.weigh(s, pop, sl2);
    pv16<D>(pop, kt + CT, voff, rs.oacc);
    wait_vmcnt_lds_idle<2 * NU*(kStages - 1)>(); // and has been read: the stage takes the wave's next but one
    seen[0] = seen[1];
    const int next = c + kStages * kWaves;
    seen[1] = seen_of(next);
    fetch(st, next, seen[1]);
    st ^= 1;
  }
  wait_vmcnt_lds_idle<0>();

  // the waves' states: O in the wave's stages, then every lane some channels of a row
  const float l_tot = quad_sum(rs.l_part[0]), l_all = LSE ? quad_sum(rs.l_full[0]) : l_tot;
  float* o = reinterpret_cast<float*>(mine);
#pragma unroll
  for (int dt = 0; dt < G16::DT; ++dt) *reinterpret_cast<f32x4*>(o + i * D + dt * 16 + 4 * g) = rs.oacc[dt][0];
  if (g == 0) {
    ms[w][i] = rs.m_ref[0];
    ls[w][i] = l_tot;
    lf[w][i] = l_all;
  }
  __syncthreads();
  for (int e = threadIdx.x; e < a.R * (D / 4); e += kThreads) {
    const int r = e / (D / 4), d = (e - r * (D / 4)) * 4;
    float m = ms[0][r];
#pragma unroll
    for (int x = 1; x < kWaves; ++x) m = fmaxf(m, ms[x][r]);
    float l = 0.0f, all = 0.0f;
    f32x4 sum = {};
#pragma unroll
    for (int x = 0; x < kWaves; ++x) {
      const float f = __builtin_amdgcn_exp2f(ms[x][r] - m);
      l = fmaf(f, ls[x][r], l);
      all = fmaf(f, lf[x][r], all);
      const f32x4 part = *reinterpret_cast<const f32x4*>(reinterpret_cast<const float*>(&Ts[x][0][0][0]) + r * D + d);
#pragma unroll
      for (int j = 0; j < 4; ++j) sum[j] = fmaf(f, part[j], sum[j]);
    }
    if (a.splits > 1) {
      const int64_t at = (bh * a.splits + it.split) * a.R + r;
      *reinterpret_cast<f32x4*>(a.part + at * D + d) = sum;
      if (d == 0) {
        a.stat[at] = make_float2(m, l);
        if constexpr (LSE) a.stat_l[at] = all;
      }
      continue;
    }
    const bool has = l > 0.0f || l != l;
    const float inv = has ? 1.0f / l : 0.0f;
    uint16_t* to = static_cast<uint16_t*>(a.out.p) + row_offset(a.out, it.b, it.kvh * a.G, r, a.N, a.G);
    const bf16x2 x = cvt2(sum[0] * inv, sum[1] * inv), y = cvt2(sum[2] * inv, sum[3] * inv);
    *reinterpret_cast<bf16x4*>(to + d) = bf16x4{x[0], x[1], y[0], y[1]};
    if constexpr (LSE) {
      if (d == 0) a.lse[bh * a.R + r] = has ? (m + __log2f(all)) * 0.69314718055994530942f : -INFINITY;
    }
  }
}

// Joins the parts of a row: O = sum of 2^(m_s - m) O_s over the same of l_s.  W waves a
// row, a run of parts each, then those in order.
template <int D, bool LSE, int W>
__global__ __launch_bounds__(kThreads) void cross_join_kernel(CrossArgs a) {
  __shared__ float os[4][128], ls[4], lf[4], ms[4];
  const int lane = threadIdx.x & 63, w = threadIdx.x >> 6, x0 = w % W;
  const int64_t row = (int64_t)blockIdx.x * (4 / W) + w / W;
  if (row >= (int64_t)a.B * a.Hkv * a.R) return;       // (W = 1 only: no barrier follows)
  const int bh = (int)(row / a.R), r = (int)(row - (int64_t)bh * a.R);
  const int b = bh / a.Hkv, kvh = bh - b * a.Hkv;
  const int s0 = a.splits * x0 / W, s1 = a.splits * (x0 + 1) / W;
  const int64_t at = (int64_t)bh * a.splits * a.R + r;

  float m = -3e38f;
#pragma unroll 4
  for (int s = s0; s < s1; ++s) m = fmaxf(m, a.stat[at + (int64_t)s * a.R].x);
  float l = 0.0f, lall = 0.0f, o0 = 0.0f, o1 = 0.0f;
#pragma unroll 4
  for (int s = s0; s < s1; ++s) {
    const int64_t j = at + (int64_t)s * a.R;
    const float2 st = a.stat[j];
    const float f = __builtin_amdgcn_exp2f(st.x - m);
    l = fmaf(f, st.y, l);
    if constexpr (LSE) lall = fmaf(f, a.stat_l[j], lall);
    if (2 * lane < D) {
      const float2 o = *reinterpret_cast<const float2*>(a.part + j * D + 2 * lane);
      o0 = fmaf(f, o.x, o0);
      o1 = fmaf(f, o.y, o1);
    }
  }
  if constexpr (W > 1) {
    os[w][2 * lane] = o0;
    os[w][2 * lane + 1] = o1;
    if (lane == 0) {
      ls[w] = l;
      lf[w] = lall;
      ms[w] = m;
    }
    __syncthreads();
    if (w != 0) return;
    m = ms[0];
#pragma unroll
    for (int x = 1; x < W; ++x) m = fmaxf(m, ms[x]);
    l = lall = o0 = o1 = 0.0f;
#pragma unroll
    for (int x = 0; x < W; ++x) {
      const float f = __builtin_amdgcn_exp2f(ms[x] - m);
      l = fmaf(f, ls[x], l);
      lall = fmaf(f, lf[x], lall);
      o0 = fmaf(f, os[x][2 * lane], o0);
      o1 = fmaf(f, os[x][2 * lane + 1], o1);
    }
  }
  const bool has = l > 0.0f || l != l;
  const float inv = has ? 1.0f / l : 0.0f;
  if (2 * lane < D) {
    uint16_t* o = static_cast<uint16_t*>(a.out.p) + row_offset(a.out, b, kvh * a.G, r, a.N, a.G);
    *reinterpret_cast<bf16x2*>(o + 2 * lane) = cvt2(o0 * inv, o1 * inv);
  }
  if constexpr (LSE) {
    if (lane == 0)
      a.lse[((int64_t)b * a.H + kvh * a.G) * a.N + r] = has ? (m + __log2f(lall)) * 0.69314718055994530942f : -INFINITY;
  }
}

constexpr int kWaveParts = 8;    // parts that one wave joins

// An entry's mask and length as bits, a word for each tile of 32 keys, and its keys up to
// the last seen one.  One workgroup an entry, a word a lane at a time.
constexpr int kBitThreads = 1024;
__global__ __launch_bounds__(kBitThreads) void cross_bits_kernel(CrossArgs a) {
  typedef unsigned __attribute__((ext_vector_type(4), aligned(1))) mask16;
  __shared__ int last[kBitThreads / 64];
  const int b = blockIdx.x, M = a.M, words = (M + 31) / 32;
  const uint8_t* mask = a.mask + b * a.mask_b;
  const int len = a.lens ? min(max(a.lens[b], 0), M) : M;
  uint32_t* bits = a.bits + (int64_t)b * words;
  int end = 0;
  for (int i = threadIdx.x; i < words; i += kBitThreads) {
    const int key = i * 32;
    uint32_t word = 0;
    if (key + 32 <= M) {
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        const mask16 x = *reinterpret_cast<const mask16*>(mask + key + 16 * h);
#pragma unroll
        for (int e = 0; e < 16; ++e) word |= ((x[e / 4] >> (8 * (e % 4))) & 255u) != 0 ? 1u << (16 * h + e) : 0u;
      }
    } else {
      for (int e = 0; key + e < M; ++e) word |= mask[key + e] != 0 ? 1u << e : 0u;
    }
    word &= rows_left(len - key);
    bits[i] = word;
    if (word) end = key + 32 - __clz(word);
  }
#pragma unroll
  for (int d = 32; d > 0; d /= 2) end = max(end, __shfl_xor(end, d));
  if (threadIdx.x % 64 == 0) last[threadIdx.x / 64] = end;
  __syncthreads();
  if (threadIdx.x == 0) {
    for (int j = 1; j < kBitThreads / 64; ++j) end = max(end, last[j]);
    a.seen[b] = end;
  }
}

template <int D, int QT>
void launch_qt(const CrossArgs& a, hipStream_t stream) {
  auto go = [&](auto kernel) { hipLaunchKernelGGL(kernel, dim3(a.wgs), dim3(kThreads), 0, stream, a); };
  if (a.mask && a.lse) go(cross_attn_kernel<D, QT, true, true>);
  else if (a.mask) go(cross_attn_kernel<D, QT, true, false>);
  else if (a.lse) go(cross_attn_kernel<D, QT, false, true>);
  else go(cross_attn_kernel<D, QT, false, false>);
}

template <int D>
void launch_d(const CrossArgs& a, const CrossShape& s, hipStream_t stream) {
  auto few = [&](auto kernel) { hipLaunchKernelGGL(kernel, dim3(a.wgs), dim3(kThreads), 0, stream, a); };
  if (s.few) {
    if (a.mask && a.lse) few(cross_few_kernel<D, true, true>);
    else if (a.mask) few(cross_few_kernel<D, true, false>);
    else if (a.lse) few(cross_few_kernel<D, false, true>);
    else few(cross_few_kernel<D, false, false>);
  } else if (s.narrow) launch_qt<D, 1>(a, stream);
  else launch_qt<D, 2>(a, stream);
  if (a.splits == 1) return;
  auto join = [&](auto kernel, int waves) {
    const int64_t rows = (int64_t)a.B * a.Hkv * a.R;
    hipLaunchKernelGGL(kernel, dim3((unsigned)((rows * waves + 3) / 4)), dim3(kThreads), 0, stream, a);
  };
  if (a.splits > kWaveParts) {
    if (a.lse) join(cross_join_kernel<D, true, 4>, 4);
    else join(cross_join_kernel<D, false, 4>, 4);
  } else {
    if (a.lse) join(cross_join_kernel<D, true, 1>, 1);
    else join(cross_join_kernel<D, false, 1>, 1);
  }
}

}  // namespace

static size_t up256(size_t x) { return (x + 255) / 256 * 256; }

// Expected microseconds of a call with row tiles of 64 (narrow) or 128 and its keys divided
// into parts.  A step over 32 keys takes a lone workgroup of a CU 0.85 us (narrow: 0.66) and
// several 0.55 (0.43) each, 0.66 and 0.38 (0.51 and 0.30) with heads of 64; what parts add is
// a launch and their results written and read.  Fitted to 240 calls of 32 to 32,768 rows over
// 64 to 16,384 keys with every shape and up to 32 parts: the shape with the least cost takes
// 1.01 times the best one's time in the geometric mean and 1.16 times at most.  Parts that
// fill the card at any cost took 1.10 and 1.87 times: 32 heads of 512 rows over 512 keys
// 28.5 us instead of 16, over 4,000 keys in narrow tiles 76.5 instead of 55 in wide ones.
static float shape_cost(bool narrow, int64_t wgs, int64_t rows, int M, int D, int splits) {
  const float lone = D == 64 ? (narrow ? 0.51f : 0.66f) : narrow ? 0.66f : 0.85f;
  const float each = D == 64 ? (narrow ? 0.30f : 0.38f) : narrow ? 0.43f : 0.55f;
  const int64_t per_cu = (wgs * splits + 255) / 256, steps = ((M + 31) / 32 + splits - 1) / splits;
  float us = (float)steps * fmaxf(lone, (float)per_cu * each);
  if (splits > 1) us += 3.3f + (float)rows * (float)(splits * D) * 8.0f / 3.6e6f;
  return us;
}

CrossShape cross_shape(int B, int Hkv, int G, int N, int M, int D, bool mask, bool grad) {
  CrossShape s{};
  const int64_t heads = (int64_t)B * Hkv, R = (int64_t)G * N;
  s.few = !grad && R <= 16;
  s.splits = 1;
  int64_t wgs = heads, places = wide_per_cu(D) * 256;   // workgroups; those that the card holds
  if (s.few) {
    // A single token's keys fill the card once (31 x 32 heads of 4,000 keys: 170 us, parts for
    // twice or three times as many workgroups 195 and 211), in parts of 128 keys or more, a
    // tile a wave.  Up to 512 keys (64 channels: 1,024) are read sooner than parts are
    // joined: 4 x 20 heads of 64 over 512 keys take 6.4 us, in 6 parts 10.9.
    s.narrow = s.tiles = 1;
    if ((int64_t)M * D > 65536 && wgs < 256) {
      const int64_t parts = 256 / wgs, most = (M + 127) / 128;
      s.splits = (int)(parts < most ? parts : most);
    }
  } else {
    float best = INFINITY;
    for (int narrow = 0; narrow < 2; ++narrow) {
      const int64_t tiles = (R + (narrow ? 63 : 127)) / (narrow ? 64 : 128);
      for (int splits = 1; splits <= 64; splits += splits < 4 ? 1 : splits & (splits - 1) ? splits / 3 : splits / 2) {
        if (splits > 1 && (heads * tiles * splits > places || M < 64 * splits)) break;
        const float us = shape_cost(narrow, heads * tiles, heads * R, M, D, splits);
        if (us >= best) continue;
        best = us;
        s.narrow = narrow;
        s.tiles = (int)tiles;
        s.splits = splits;
      }
    }
    wgs = heads * s.tiles;
  }
  // Runs of row tiles, for which K and V are found and Q comes ahead, where the card is filled
  // four times over: 63,240 rows of 32 heads over 512 keys 680 us, in runs of up to 16 and two
  // rounds 796.
  const int64_t run = wgs / (4 * places);
  s.run = (int)(run < 1 ? 1 : run < 8 ? run : 8);
  size_t at = 0;
  if (mask) {
    s.bits_at = at;
    at += up256((size_t)B * ((M + 31) / 32) * 4);
    s.seen_at = at;
    at += up256((size_t)B * 4);
  }
  if (s.splits > 1) {
    const size_t rows = (size_t)heads * s.splits * R;
    s.stat_at = at;
    at += up256(rows * 8);
    s.stat_l_at = at;
    at += up256(rows * 4);
    s.part_at = at;
    at += up256(rows * D * 4);
  }
  s.ws_bytes = at;
  return s;
}

hipError_t launch_cross_bits(const CrossArgs& a, hipStream_t stream) {
  hipLaunchKernelGGL(cross_bits_kernel, dim3(a.B), dim3(kBitThreads), 0, stream, a);
  return hipGetLastError();
}

hipError_t launch_cross_attention(const CrossArgs& a, const CrossShape& s, hipStream_t stream) {
  if (a.mask) {
    const hipError_t e = launch_cross_bits(a, stream);
    if (e != hipSuccess) return e;
  }
  if (a.D == 64) launch_d<64>(a, s, stream);
  else if (a.D == 112) launch_d<112>(a, s, stream);
  else launch_d<128>(a, s, stream);
  return hipGetLastError();
}

}  // namespace sva
