// Gradients of cross attention.  With P = exp(c s - lse), dO the gradient of O and
// delta = rowsum(dO O):
//   dV = P^T dO, dP = dO V^T, dS = P (dP - delta), dQ = c dS K, dK = c dS^T Q.
//
// Two launches, so that no sum goes through atomics and the same call gives the same
// bits; S and dP are formed in both (seven products where five would do, against
// partial dQ of every key tile through memory).
//   rows: a workgroup holds 128 (64) rows, as the forward kernel does, with Q and dO
//     in registers, and walks the keys; P and dS stay in registers and are the operands
//     of dQ^T += K^T dS^T and of (P K)^T as they stand.  It forms delta from out, which
//     was rounded to bf16: what the dS of a row then sum to instead of zero, e, is given
//     back, as dQ = c (dS K - e P K), and to the second launch as delta + e.  Without it
//     dQ and dK of rows with one large weight were off by up to three times what their
//     own rounding takes; P K costs an eighth of the call (63,240 rows of 32 heads over
//     512 keys 2,305 us instead of 2,060), O formed again in place of e more.
//   keys: a workgroup holds 128 keys (32 a wave) with K and V in registers and walks
//     the rows of all heads of the group, so dK and dV are summed over them where they
//     are; S = Q K^T here has the rows in the registers and a key in every lane, P and
//     dS are again operands as they stand.  The walk is divided among workgroups where
//     keys are few, and the parts are added in order by a third launch.
// P and dS are rounded to bf16 once, for their products; everything else is float32.
//
// Bound as the forward kernel is.  63,240 rows of 32 heads of 128 over 512 keys: rows 1,290
// us, keys 970, the parts' sum 13; 920 TFLOP/s over the eight products.
#include "cross_tiles.h"

namespace sva {
namespace {

using namespace cross;

constexpr int NST = 4, PD = 3;   // LDS stages, tiles ahead

template <int D, int QT, bool MASK>
__global__ __launch_bounds__(kThreads) __attribute__((amdgpu_waves_per_eu(wide_per_cu(D), QT == 2 ? wide_per_cu(D) : 4)))
void cross_grad_rows_kernel(CrossArgs a) {
  using G16 = Geo16<D>;
  using Feed = KeyFeed<D, MASK, true>;
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

  // Q and dO of the wave's rows, their lse and delta.  (Loads of the next rows' during a
  // tile's last product would keep 32 to 96 more registers alive beside both sums: 63,240
  // rows over 512 keys 2,670 and 3,190 us instead of 2,305.)
  bf16x8 qop[QT][G16::KS], gop[QT][G16::KS];
  float lse2[QT], delta[QT], excess[QT];
  bf16x8 oop[QT][G16::KS];
  float lse[QT];
  auto take_rows = [&](int tile) {
    const uint16_t *qrow[QT], *grow[QT];
#pragma unroll
    for (int qt = 0; qt < QT; ++qt) {
      const int r = row_of(tile, qt);
      qrow[qt] = grow[qt] = nullptr;
      lse[qt] = -INFINITY;
      if (r < a.R) {
        qrow[qt] = static_cast<const uint16_t*>(a.q.p) + row_offset(a.q, it.b, it.kvh * a.G, r, a.N, a.G);
        grow[qt] = static_cast<const uint16_t*>(a.dout.p) + row_offset(a.dout, it.b, it.kvh * a.G, r, a.N, a.G);
        lse[qt] = a.lse[bh * a.R + r];
      }
    }
    load_operand<D>(qop, qrow, lane);
    load_operand<D>(gop, grow, lane);
    const uint16_t* orow[QT];
#pragma unroll
    for (int qt = 0; qt < QT; ++qt) {
      const int r = row_of(tile, qt);
      orow[qt] = r < a.R ? static_cast<const uint16_t*>(a.out.p) + row_offset(a.out, it.b, it.kvh * a.G, r, a.N, a.G) : nullptr;
    }
    load_operand<D>(oop, orow, lane);
#pragma unroll
    for (int qt = 0; qt < QT; ++qt) {
      float s = 0.0f;
#pragma unroll
      for (int x = 0; x < G16::KS; ++x)
#pragma unroll
        for (int e = 0; e < 8; ++e) s = fmaf((float)gop[qt][x][e], (float)oop[qt][x][e], s);
      delta[qt] = quad_sum(s);
      // a row that saw no key has P = 0 everywhere
      lse2[qt] = lse[qt] == -INFINITY ? INFINITY : lse[qt] * 1.4426950408889634074f;
      excess[qt] = 0.0f;
    }
  };
  // A row's dS sum to zero but for e, what out's rounding to bf16 took from delta: e is given
  // back to delta for the second launch, and dQ is dS K - e P K.
  f32x4 dq[G16::DT][QT] = {}, pk[G16::DT][QT] = {};
  auto store = [&](int tile) {
#pragma unroll
    for (int qt = 0; qt < QT; ++qt) {
      const int r = row_of(tile, qt);
      const float e = quad_sum(excess[qt]);
      if (a.splits > 1) {
        if (r < a.R) {
          const int64_t at = (bh * a.splits + it.split) * a.R + r;
          float* o = a.part + at * (2 * D);
#pragma unroll
          for (int dt = 0; dt < G16::DT; ++dt) {
            *reinterpret_cast<f32x4*>(o + dt * 16 + 4 * g) = dq[dt][qt];
            *reinterpret_cast<f32x4*>(o + D + dt * 16 + 4 * g) = pk[dt][qt];
          }
          if (g == 0) {
            a.stat_l[at] = e;
            if (it.split == 0) a.stat[bh * a.R + r] = make_float2(lse2[qt], delta[qt]);
          }
        }
      } else {
        uint16_t* o = r < a.R ? static_cast<uint16_t*>(a.dq.p) + row_offset(a.dq, it.b, it.kvh * a.G, r, a.N, a.G) : nullptr;
#pragma unroll
        for (int dt = 0; dt < G16::DT; ++dt)
#pragma unroll
          for (int j = 0; j < 4; ++j) dq[dt][qt][j] = fmaf(-e, pk[dt][qt][j], dq[dt][qt][j]);
        store_row<D>(o, &dq[0][qt], QT, a.scale, g);
        if (g == 0 && r < a.R) a.stat[bh * a.R + r] = make_float2(lse2[qt], delta[qt] + e);
      }
#pragma unroll
      for (int dt = 0; dt < G16::DT; ++dt) dq[dt][qt] = pk[dt][qt] = f32x4{};
    }
  };

  if (it.chunks == 0) {            // no key: zeros
    for (int t = 0; t < it.tiles; ++t) {
      take_rows(it.tile + t);      // (other parts may have keys)
      store(it.tile + t);
    }
    return;
  }
  Feed feed;
  feed.start(a, it, w, lane);
  feed.ld.clear_pads(&Ks[0][0], NST);
  feed.ld.clear_pads(&Vs[0][0], NST);
  auto fetch = [&](int st) { return feed.feed(a, ks_base + st * CT, vs_base + st * CT); };
  uint32_t seen[PD];               // which keys of the tiles ahead are
#pragma unroll
  for (int c = 0; c < PD; ++c) seen[c] = fetch(c);
  take_rows(it.tile);

  const Places<D> at(lane);
  int st = 0, c = 0, tile = it.tile;
  const int end = it.tile + it.tiles;
#pragma unroll 1
  while (true) {
    wait_vmcnt_lds_idle<Feed::kLoads * (PD - 1)>();    // the tile has landed
    wg_barrier();                                      // and every wave is done with the one before
    const uint32_t fed = fetch((st + PD) % NST);
    const unsigned kt = ks_base + st * CT, vt = vs_base + st * CT;
    u32x4 pw[QT], dsw[QT];
    // 16 keys at a time: 16 registers of S and dP are alive beside dQ and P K, not 32
#pragma unroll
    for (int x = 0; x < 2; ++x) {
      f32x4 s[QT], dp[QT];
      rows_times_half<D, QT>(s, kt + x * 16 * Geo<D>::RB, at, qop);
      rows_times_half<D, QT>(dp, vt + x * 16 * Geo<D>::RB, at, gop);
      // Vector instructions may read a product eight wait states after its last instruction.
      // Where the branch below comes between, the compiler has left them out (heads of 64, 16
      // rows a wave), and S was read before it was there.
      settle(s, dp);
      if (__builtin_expect(seen[0] != ~0u, 0)) {
        asm volatile("");
        const uint32_t mine = seen[0] >> (16 * x + 4 * g);
#pragma unroll
        for (int r = 0; r < 4; ++r)
          if (!(mine >> r & 1)) {
#pragma unroll
            for (int qt = 0; qt < QT; ++qt) s[qt][r] = -INFINITY;
          }
      }
#pragma unroll
      for (int qt = 0; qt < QT; ++qt)
#pragma unroll
        for (int e = 0; e < 2; ++e) {
          const float p0 = __builtin_amdgcn_exp2f(__builtin_fmaf(s[qt][2 * e], sl2, -lse2[qt]));
          const float p1 = __builtin_amdgcn_exp2f(__builtin_fmaf(s[qt][2 * e + 1], sl2, -lse2[qt]));
          const float d0 = p0 * (dp[qt][2 * e] - delta[qt]), d1 = p1 * (dp[qt][2 * e + 1] - delta[qt]);
          excess[qt] += d0 + d1;
          pw[qt][x * 2 + e] = __builtin_bit_cast(unsigned, cvt2(p0, p1));
          dsw[qt][x * 2 + e] = __builtin_bit_cast(unsigned, cvt2(d0, d1));
        }
    }
#pragma unroll
    for (int x = 1; x < PD; ++x) seen[x - 1] = seen[x];
    seen[PD - 1] = fed;
    bf16x8 pop[QT], dsop[QT];
#pragma unroll
    for (int qt = 0; qt < QT; ++qt) {
      pop[qt] = __builtin_bit_cast(bf16x8, pw[qt]);
      dsop[qt] = __builtin_bit_cast(bf16x8, dsw[qt]);
    }
    cols_times_both<D, QT>(dsop, pop, kt, at, dq, pk);
    st = (st + 1) % NST;
    if (++c == it.chunks) {
      store(tile);
      c = 0;
      if (++tile == end) break;
      take_rows(tile);
    }
  }
  wait_vmcnt<0>();                 // no load may still target this workgroup's LDS
}

template <int D>
__global__ __launch_bounds__(kThreads) __attribute__((amdgpu_waves_per_eu(2, 2)))
void cross_grad_keys_kernel(CrossArgs a) {
  using G16 = Geo16<D>;
  using Loader = TileLoader<D>;
  constexpr int CT = Loader::CT, NUW = Loader::NUW, KT = 2;
  constexpr int kLoads = 2 * NUW + 1;            // of a wave for a tile: Q, dO, statistics
  __shared__ __attribute__((aligned(1024))) unsigned char Qs[NST][CT];
  __shared__ __attribute__((aligned(1024))) unsigned char Gs[NST][CT];
  __shared__ __attribute__((aligned(256))) float2 Ss[NST][CK];

  const int lane = threadIdx.x & 63, i = lane & 15, g = lane >> 4;
  const int w = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  // part of the rows, key tile, kv head of an entry (the fastest, as in the other kernels)
  const int heads = a.B * a.Hkv, part = blockIdx.x / heads, bh = blockIdx.x - part * heads;
  const int split = part / a.key_tiles, tile = part - split * a.key_tiles;
  const int b = bh / a.Hkv, kvh = bh - b * a.Hkv;
  const int count = seen_keys_of_all(a, b);
  const int key0 = tile * 128 + w * 32;
  const float sl2 = a.scale_log2;

  f32x4 dk[G16::DT][KT] = {}, dv[G16::DT][KT] = {};
  if (tile * 128 < count) {
    bf16x8 kop[KT][G16::KS], vop[KT][G16::KS];
    {
      const uint16_t *krow[KT], *vrow[KT];
#pragma unroll
      for (int kt = 0; kt < KT; ++kt) {
        const int j = key0 + kt * 16 + i;
        krow[kt] = vrow[kt] = nullptr;
        if (is_seen(a, b, j, count)) {
          krow[kt] = static_cast<const uint16_t*>(a.k.p) + b * a.k.sb + kvh * a.k.sh + j * a.k.sn;
          vrow[kt] = static_cast<const uint16_t*>(a.v.p) + b * a.v.sb + kvh * a.v.sh + j * a.v.sn;
        }
      }
      load_operand<D>(kop, krow, lane);
      load_operand<D>(vop, vrow, lane);
    }

    // The walk: tiles of 32 tokens of the group's first head, then of the next.
    const int per_head = (a.N + CK - 1) / CK;
    const int64_t all = (int64_t)per_head * a.G;
    const int64_t t0 = all * split / a.row_splits, t1 = all * (split + 1) / a.row_splits;
    Loader ld;
    ld.init(w, lane);
    const unsigned qs_base = __builtin_amdgcn_readfirstlane((unsigned)(size_t)(const lds_u8*)&Qs[0][0]);
    const unsigned gs_base = __builtin_amdgcn_readfirstlane((unsigned)(size_t)(const lds_u8*)&Gs[0][0]);
    const unsigned ss_base = __builtin_amdgcn_readfirstlane((unsigned)(size_t)(const lds_u8*)&Ss[0][0]);
    ld.clear_pads(&Qs[0][0], NST);
    ld.clear_pads(&Gs[0][0], NST);
    int64_t ft = t0;                             // the next tile to load
    int fh = (int)(t0 / per_head), fn = (int)(t0 - (int64_t)fh * per_head) * CK;
    const uint16_t *qp, *gp;
    const float2* sp;
    auto bases = [&]() {
      const int64_t h = kvh * a.G + (ft < t1 ? fh : 0);
      qp = static_cast<const uint16_t*>(a.q.p) + b * a.q.sb + h * a.q.sh + fn * a.q.sn;
      gp = static_cast<const uint16_t*>(a.dout.p) + b * a.dout.sb + h * a.dout.sh + fn * a.dout.sn;
      sp = a.stat + ((int64_t)b * a.H + h) * a.N + fn;
    };
    bases();
    uint32_t qoff[NUW], goff[NUW];
    ld.offsets(a.q.sn, qoff);
    ld.offsets(a.dout.sn, goff);
    auto fetch = [&](int st) {
      const int left = ft < t1 ? a.N - fn : 0;
      ld.load(qp, a.q.sn, qoff, rows_left(left), qs_base + st * CT);
      ld.load(gp, a.dout.sn, goff, rows_left(left), gs_base + st * CT);
      const float* from = reinterpret_cast<const float*>(sp) + lane;
      global_to_lds<4>(lane / 2 < left ? from : kInf + (lane & 1), ss_base + st * (int)(CK * sizeof(float2)));
      ++ft;
      fn += CK;
      qp += CK * a.q.sn;
      gp += CK * a.dout.sn;
      sp += CK;
      if (fn >= a.N) {
        fn = 0;
        ++fh;
        bases();
      }
    };
    const Places<D> at(lane);
#pragma unroll
    for (int c = 0; c < PD; ++c) fetch(c);
    int st = 0;
#pragma unroll 1
    for (int64_t t = t0; t < t1; ++t) {
      wait_vmcnt_lds_idle<kLoads * (PD - 1)>();      // this tile has landed
      wg_barrier();                                  // and every wave is done with the one before
      fetch((st + PD) % NST);
      if (key0 < count) {
        const unsigned qt = qs_base + st * CT, gt = gs_base + st * CT;
        const float4* stat = reinterpret_cast<const float4*>(&Ss[st][0]);   // rows 2x and 2x + 1
        // half a tile's rows at a time: S and dP of all 32 would crowd out what is read ahead
        bf16x8 pop[KT], dsop[KT];
        u32x4 pw[KT], dw[KT];
#pragma unroll
        for (int x = 0; x < 2; ++x) {
          f32x4 s[KT], dp[KT];
          rows_times_half<D>(s, qt + x * 16 * Geo<D>::RB, at, kop);
          rows_times_half<D>(dp, gt + x * 16 * Geo<D>::RB, at, vop);
#pragma unroll
          for (int e = 0; e < 2; ++e) {
            const float4 z = stat[x * 8 + 2 * g + e];      // (lse, delta) of two rows
#pragma unroll
            for (int kt = 0; kt < KT; ++kt) {
              const float p0 = __builtin_amdgcn_exp2f(__builtin_fmaf(s[kt][2 * e], sl2, -z.x));
              const float p1 = __builtin_amdgcn_exp2f(__builtin_fmaf(s[kt][2 * e + 1], sl2, -z.z));
              pw[kt][x * 2 + e] = __builtin_bit_cast(unsigned, cvt2(p0, p1));
              dw[kt][x * 2 + e] = __builtin_bit_cast(unsigned, cvt2(p0 * (dp[kt][2 * e] - z.y), p1 * (dp[kt][2 * e + 1] - z.w)));
            }
          }
        }
#pragma unroll
        for (int kt = 0; kt < KT; ++kt) {
          pop[kt] = __builtin_bit_cast(bf16x8, pw[kt]);
          dsop[kt] = __builtin_bit_cast(bf16x8, dw[kt]);
        }
        cols_times<D>(pop, gt, at, dv);
        cols_times<D>(dsop, qt, at, dk);
      }
      st = (st + 1) % NST;
    }
    wait_vmcnt<0>();               // no load may still target this workgroup's LDS
  }

#pragma unroll
  for (int kt = 0; kt < KT; ++kt) {
    const int j = key0 + kt * 16 + i;
    if (a.row_splits > 1) {
      if (j >= count) continue;                  // the join knows which are hidden
      float* k = a.part_kv + ((((int64_t)bh * a.row_splits + split) * 2) * a.M + j) * D;
      float* v = k + (int64_t)a.M * D;
#pragma unroll
      for (int dt = 0; dt < G16::DT; ++dt) {
        *reinterpret_cast<f32x4*>(k + dt * 16 + 4 * g) = dk[dt][kt];
        *reinterpret_cast<f32x4*>(v + dt * 16 + 4 * g) = dv[dt][kt];
      }
      continue;
    }
    if (!is_seen(a, b, j, count)) {              // a hidden key's gradients are zeros
#pragma unroll
      for (int dt = 0; dt < G16::DT; ++dt) dk[dt][kt] = dv[dt][kt] = f32x4{};
    }
    uint16_t *k = nullptr, *v = nullptr;
    if (j < a.M) {
      k = static_cast<uint16_t*>(a.dk.p) + b * a.dk.sb + kvh * a.dk.sh + j * a.dk.sn;
      v = static_cast<uint16_t*>(a.dv.p) + b * a.dv.sb + kvh * a.dv.sh + j * a.dv.sn;
    }
    store_row<D>(k, &dk[0][kt], KT, a.scale, g);
    store_row<D>(v, &dv[0][kt], KT, 1.0f, g);
  }
}

// Adds the parts of dQ (which 0: of dS K, P K and e, and delta gets e) or of dK and dV (1,
// 2) in their order, four channels a lane; a hidden key's gradients are zeros.
template <int D>
__global__ __launch_bounds__(kThreads) void cross_sum_kernel(CrossArgs a, int first) {
  constexpr int kLanes = D / 4, kRows = kThreads / kLanes;
  const int which = first + blockIdx.y, c = threadIdx.x % kLanes * 4;
  const int rows = which == 0 ? a.R : a.M, parts = which == 0 ? a.splits : a.row_splits;
  const int64_t at = (int64_t)blockIdx.x * kRows + threadIdx.x / kLanes;
  if (threadIdx.x >= kRows * kLanes || at >= (int64_t)a.B * a.Hkv * rows) return;
  const int bh = (int)(at / rows), r = (int)(at - (int64_t)bh * rows);
  const int b = bh / a.Hkv, kvh = bh - b * a.Hkv;
  f32x4 s = {};
  if (which == 0) {
    const int64_t first_part = (int64_t)bh * parts * rows + r;
    f32x4 pk = {};
    float e = 0.0f;
#pragma unroll 4
    for (int p = 0; p < parts; ++p) {
      const int64_t x = first_part + (int64_t)p * rows;
      s += *reinterpret_cast<const f32x4*>(a.part + x * (2 * D) + c);
      pk += *reinterpret_cast<const f32x4*>(a.part + x * (2 * D) + D + c);
      e += a.stat_l[x];
    }
#pragma unroll
    for (int j = 0; j < 4; ++j) s[j] = fmaf(-e, pk[j], s[j]);
    if (c == 0) a.stat[at].y += e;
  } else if (is_seen(a, b, r, seen_keys(a, b))) {
    const float* from = a.part_kv + (((int64_t)bh * parts * 2 + (which - 1)) * rows + r) * D + c;
    const int64_t step = (int64_t)rows * D * 2;
#pragma unroll 4
    for (int p = 0; p < parts; ++p) s += *reinterpret_cast<const f32x4*>(from + p * step);
  }
  const float f = which == 2 ? 1.0f : a.scale;
  const bf16x2 x = cvt2(s[0] * f, s[1] * f), y = cvt2(s[2] * f, s[3] * f);
  const bf16x4 z = {x[0], x[1], y[0], y[1]};
  int64_t off;
  const HeadsView& to = which == 0 ? a.dq : which == 1 ? a.dk : a.dv;
  if (which == 0) off = row_offset(to, b, kvh * a.G, r, a.N, a.G);
  else off = b * to.sb + kvh * to.sh + r * to.sn;
  *reinterpret_cast<bf16x4*>(static_cast<uint16_t*>(to.p) + off + c) = z;
}

template <int D>
void launch_d(const CrossArgs& a, const CrossShape& s, hipStream_t stream) {
  auto go = [&](auto kernel, int wgs) { hipLaunchKernelGGL(kernel, dim3(wgs), dim3(kThreads), 0, stream, a); };
  if (s.narrow && a.mask) go(cross_grad_rows_kernel<D, 1, true>, a.wgs);
  else if (s.narrow) go(cross_grad_rows_kernel<D, 1, false>, a.wgs);
  else if (a.mask) go(cross_grad_rows_kernel<D, 2, true>, a.wgs);
  else go(cross_grad_rows_kernel<D, 2, false>, a.wgs);
  auto sum = [&](int first, int n, int64_t rows) {
    constexpr int kRows = kThreads / (D / 4);
    hipLaunchKernelGGL(cross_sum_kernel<D>, dim3((unsigned)((rows + kRows - 1) / kRows), n), dim3(kThreads), 0, stream, a, first);
  };
  if (a.splits > 1) sum(0, 1, (int64_t)a.B * a.Hkv * a.R);
  go(cross_grad_keys_kernel<D>, a.kv_wgs);
  if (a.row_splits > 1) sum(1, 2, (int64_t)a.B * a.Hkv * a.M);
}

size_t up256(size_t x) { return (x + 255) / 256 * 256; }

}  // namespace

CrossShape cross_grad_shape(int B, int Hkv, int G, int N, int M, int D, bool mask) {
  CrossShape s = cross_shape(B, Hkv, G, N, M, D, mask, true);
  const int64_t heads = (int64_t)B * Hkv, R = (int64_t)G * N;
  s.key_tiles = (M + 127) / 128;
  const int64_t base = heads * s.key_tiles, walk = (((int64_t)N + 31) / 32 * G + 7) / 8;
  // The rows of a tile of keys are divided where that is worth its partial sums: a step over
  // 32 rows takes a lone workgroup of a CU 1.56 us and a pair 1.95 (0.78 and 1.0 with heads of
  // 64), parts a launch and their sums written and read.  Of 139 calls (1 to 16,384 rows, 64
  // to 4,000 keys) timed with every number of parts, the one chosen took 1.003 times the best
  // one's time in the geometric mean, 1.12 at most; parts for 1,024 workgroups 1.03 and 1.34
  // (32 heads of 512 rows over 1,536 keys: 130 us instead of 96).
  const float lone = D == 64 ? 0.78f : 1.56f, pair = D == 64 ? 1.0f : 1.95f;
  float best = INFINITY;
  for (int parts = 1; parts <= 1024; parts += parts < 4 ? 1 : parts & (parts - 1) ? parts / 3 : parts / 2) {
    if (parts > 1 && (parts > walk || base * parts > 1024)) break;
    const int64_t per_cu = (base * parts + 255) / 256, steps = (((int64_t)N + 31) / 32 * G + parts - 1) / parts;
    float us = (float)steps * ((float)(per_cu / 2) * pair + (float)(per_cu % 2) * lone);
    if (parts > 1) us += 3.3f + (float)(heads * M) * (float)(parts * D) * 16.0f / 3.6e6f;
    if (us >= best) continue;
    best = us;
    s.row_splits = parts;
  }
  size_t at = mask ? s.seen_at + up256((size_t)B * 4) : 0;
  s.stat_at = at;
  at += up256((size_t)heads * R * 8);
  s.stat_l_at = at;
  if (s.splits > 1) at += up256((size_t)heads * s.splits * R * 4);
  s.part_at = at;
  if (s.splits > 1) at += up256((size_t)heads * s.splits * R * D * 8);
  s.part_kv_at = at;
  if (s.row_splits > 1) at += up256((size_t)heads * s.row_splits * 2 * M * D * 4);
  s.ws_bytes = at;
  return s;
}

hipError_t launch_cross_attention_grad(const CrossArgs& a, const CrossShape& s, hipStream_t stream) {
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
