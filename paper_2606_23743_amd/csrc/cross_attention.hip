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
// Hidden keys are not loaded at all: a length ends the walk, a mask is first turned
// into the list of the keys it leaves.  Where few rows meet many keys, the keys are
// divided among workgroups and their results joined by a second launch.
#include "cross_tiles.h"

namespace sva {
namespace {

using namespace cross;

constexpr int NST = 4, PD = 3;   // LDS stages, tiles ahead

// a row's reference moves when a logit passes it by this much (log2 units)
constexpr float kSlack = 30.0f;

template <int D, int QT, bool GATHER, bool LSE>
__global__ __launch_bounds__(kThreads) __attribute__((amdgpu_waves_per_eu(2, QT == 2 ? 2 : 4)))
void cross_attn_kernel(CrossArgs a) {
  using G16 = Geo16<D>;
  using Loader = TileLoader<D>;
  constexpr int CT = Loader::CT, NUW = Loader::NUW;
  __shared__ __attribute__((aligned(1024))) unsigned char Ks[NST][CT];
  __shared__ __attribute__((aligned(1024))) unsigned char Vs[NST][CT];
  __shared__ int ring[GATHER ? RowRing::kSize : 1];

  const int lane = threadIdx.x & 63, i = lane & 15;
  const int w = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  // (kv head of an entry, part of its keys, row tile)
  const int id = __builtin_amdgcn_readfirstlane(xcd_remap(blockIdx.x, a.wgs));
  const int per = a.tiles * a.splits, bh = id / per, rest = id - bh * per;
  const int split = rest / a.tiles, tile = rest - split * a.tiles;
  const int b = bh / a.Hkv, kvh = bh - b * a.Hkv;

  // this part's keys
  const int count = seen_keys_of_all(a, b);
  const int chunks_all = (count + CK - 1) / CK;
  const int c0 = (int)((int64_t)chunks_all * split / a.splits), c1 = (int)((int64_t)chunks_all * (split + 1) / a.splits);
  const int chunks = c1 - c0;

  const int row0 = tile * 64 * QT + w * 16 * QT;
  const uint16_t* Kh = static_cast<const uint16_t*>(a.k.p) + b * a.k.sb + kvh * a.k.sh;
  const uint16_t* Vh = static_cast<const uint16_t*>(a.v.p) + b * a.v.sb + kvh * a.v.sh;
  const float sl2 = a.scale_log2;

  Loader ld;
  ld.init(w, lane);
  const unsigned ks_base = __builtin_amdgcn_readfirstlane((unsigned)(size_t)(const lds_u8*)&Ks[0][0]);
  const unsigned vs_base = __builtin_amdgcn_readfirstlane((unsigned)(size_t)(const lds_u8*)&Vs[0][0]);
  RowRing rr{ring, GATHER ? a.rows + (int64_t)b * a.M : nullptr, count};
  // tile c0 + c into stage st; one past the part's end loads zeros, so that every step waits for as many
  auto fetch = [&](int st, int c) {
    const int first = (c0 + c) * CK, end = c < chunks ? count : 0;
    if constexpr (GATHER) {
      int list[NUW];
#pragma unroll
      for (int u = 0; u < NUW; ++u) list[u] = c < chunks ? rr.at(first + ld.row[u]) : 0;
      ld.load_rows(Kh, a.k.sn, list, end - first, ks_base + st * CT);
      ld.load_rows(Vh, a.v.sn, list, end - first, vs_base + st * CT);
    } else {
      ld.load(Kh, a.k.sn, first, end, ks_base + st * CT);
      ld.load(Vh, a.v.sn, first, end, vs_base + st * CT);
    }
  };

  bf16x8 qop[QT][G16::KS];
  const uint16_t* qrow[QT];
#pragma unroll
  for (int qt = 0; qt < QT; ++qt) {
    const int r = row0 + qt * 16 + i;
    qrow[qt] = r < a.R ? static_cast<const uint16_t*>(a.q.p) + row_offset(a.q, b, kvh * a.G, r, a.N) : nullptr;
  }
  load_operand<D>(qop, qrow, lane);

  int koff[G16::KS], voff[G16::DT];
  operand_offsets<D>(lane, koff, voff);
  float m_ref[QT], l_part[QT] = {}, l_full[QT] = {}, limit[QT];
  f32x4 oacc[G16::DT][QT] = {};
#pragma unroll
  for (int qt = 0; qt < QT; ++qt) {
    m_ref[qt] = -3e38f;
    limit[qt] = -INFINITY;
  }

  // moves the reference of rows that have a logit above their limit
  auto follow = [&](const f32x4 (&s)[2][QT]) {
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
        for (int dt = 0; dt < G16::DT; ++dt)
#pragma unroll
          for (int r = 0; r < 4; ++r) oacc[dt][qt][r] *= f;
        m_ref[qt] = m_new;
        limit[qt] = (m_new + kSlack) / sl2;
      }
    }
  };
  auto softmax = [&](const f32x4 (&s)[2][QT], bf16x8 (&pop)[QT]) {
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
  };

  if (chunks > 0) {
    if constexpr (GATHER) {
      rr.fill(c0 * CK);
      rr.fill(c0 * CK + RowRing::kHalf);
      __syncthreads();
    }
#pragma unroll
    for (int c = 0; c < PD; ++c) fetch(c, c);
    // Tile c's loads are 2 * NUW of this wave's; Q's came before them.
    wait_vmcnt<2 * NUW * (PD - 1)>();
    wg_barrier();
    f32x4 sacc[2][QT];
    qk16<D>(sacc, &Ks[0][0], koff, qop);
    if (count - c0 * CK < CK) mask_tail16(sacc, count - c0 * CK, lane);
    int st = 0;
#pragma unroll 1
    for (int c = 0; c < chunks; ++c) {
      wait_vmcnt_lds_idle<2 * NUW * (PD - 2)>();     // tile c + 1 has landed
      wg_barrier();                                  // and every wave is done with tile c - 1
      if constexpr (GATHER) {
        if (c != 0 && c % (RowRing::kHalf / CK) == 0) rr.fill(c0 * CK + c * CK + RowRing::kHalf);
      }
      fetch((st + PD) % NST, c + PD);
      follow(sacc);
      f32x4 snext[2][QT];
      bf16x8 pop[QT];
      qk16<D>(snext, &Ks[0][0] + (st + 1) % NST * CT, koff, qop);
      softmax(sacc, pop);
      __builtin_amdgcn_s_setprio(1);
      pv16<D>(pop, &Vs[0][0] + st * CT, voff, oacc);
      __builtin_amdgcn_s_setprio(0);
      const int left = __builtin_amdgcn_readfirstlane(count - (c0 + c + 1) * CK);
      if (__builtin_expect(left < CK, 0)) {
        asm volatile("");
        mask_tail16(snext, left, lane);
      }
#pragma unroll
      for (int x = 0; x < 2; ++x)
#pragma unroll
        for (int qt = 0; qt < QT; ++qt) sacc[x][qt] = snext[x][qt];
      st = (st + 1) % NST;
    }
    wait_vmcnt<0>();               // no load may still target this workgroup's LDS
  }

  const int g = lane >> 4;
#pragma unroll
  for (int qt = 0; qt < QT; ++qt) {
    const float l_tot = quad_sum(l_part[qt]);
    const float l_all = LSE ? quad_sum(l_full[qt]) : l_tot;
    const int r = row0 + qt * 16 + i;
    if (r >= a.R) continue;
    if (a.splits > 1) {
      const int64_t at = ((int64_t)bh * a.splits + split) * a.R + r;
      float* o = a.part + at * D;
#pragma unroll
      for (int dt = 0; dt < G16::DT; ++dt) *reinterpret_cast<f32x4*>(o + dt * 16 + 4 * g) = oacc[dt][qt];
      if (g == 0) {
        a.stat[at] = make_float2(m_ref[qt], l_tot);
        if constexpr (LSE) a.stat_l[at] = l_all;
      }
      continue;
    }
    const bool has = l_tot > 0.0f || l_tot != l_tot;   // a NaN stays one
    const float inv = has ? 1.0f / l_tot : 0.0f;
    uint16_t* o = static_cast<uint16_t*>(a.out.p) + row_offset(a.out, b, kvh * a.G, r, a.N);
#pragma unroll
    for (int dt = 0; dt < G16::DT; ++dt) {
      const bf16x2 x = cvt2(oacc[dt][qt][0] * inv, oacc[dt][qt][1] * inv);
      const bf16x2 y = cvt2(oacc[dt][qt][2] * inv, oacc[dt][qt][3] * inv);
      const bf16x4 z = {x[0], x[1], y[0], y[1]};
      *reinterpret_cast<bf16x4*>(o + dt * 16 + 4 * g) = z;
    }
    if constexpr (LSE) {
      if (g == 0)
        a.lse[((int64_t)b * a.H + kvh * a.G) * a.N + r] =
            has ? (m_ref[qt] + __log2f(l_all)) * 0.69314718055994530942f : -INFINITY;
    }
  }
}

// Joins the parts of a row: O = sum of 2^(m_s - m) O_s over the same of l_s.  One
// workgroup a row, its waves a run of parts each, then those in order.
template <int D, bool LSE>
__global__ __launch_bounds__(kThreads) void cross_join_kernel(CrossArgs a) {
  __shared__ float os[4][128], ls[4], lf[4], ms[4];
  const int lane = threadIdx.x & 63, w = threadIdx.x >> 6;
  const int bh = blockIdx.x / a.R, r = blockIdx.x - bh * a.R;
  const int b = bh / a.Hkv, kvh = bh - b * a.Hkv;
  const int s0 = a.splits * w / 4, s1 = a.splits * (w + 1) / 4;
  const int64_t at = (int64_t)bh * a.splits * a.R + r;

  float m = -3e38f;
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
  os[w][2 * lane] = o0;
  os[w][2 * lane + 1] = o1;
  if (lane == 0) {
    ls[w] = l;
    lf[w] = lall;
    ms[w] = m;
  }
  __syncthreads();
  if (w != 0) return;
  const float top = fmaxf(fmaxf(ms[0], ms[1]), fmaxf(ms[2], ms[3]));
  l = lall = o0 = o1 = 0.0f;
#pragma unroll
  for (int x = 0; x < 4; ++x) {
    const float f = __builtin_amdgcn_exp2f(ms[x] - top);
    l = fmaf(f, ls[x], l);
    lall = fmaf(f, lf[x], lall);
    o0 = fmaf(f, os[x][2 * lane], o0);
    o1 = fmaf(f, os[x][2 * lane + 1], o1);
  }
  const bool has = l > 0.0f || l != l;
  const float inv = has ? 1.0f / l : 0.0f;
  if (2 * lane < D) {
    uint16_t* o = static_cast<uint16_t*>(a.out.p) + row_offset(a.out, b, kvh * a.G, r, a.N);
    *reinterpret_cast<bf16x2*>(o + 2 * lane) = cvt2(o0 * inv, o1 * inv);
  }
  if constexpr (LSE) {
    if (lane == 0)
      a.lse[((int64_t)b * a.H + kvh * a.G) * a.N + r] = has ? (top + __log2f(lall)) * 0.69314718055994530942f : -INFINITY;
  }
}

// The list of an entry's keys: those that mask and length leave, in order, then the
// others, in order.  One workgroup an entry, 16 keys a lane at a time.
constexpr int kListThreads = 1024, kListKeys = 16;
__global__ __launch_bounds__(kListThreads) void cross_rows_kernel(CrossArgs a) {
  typedef unsigned __attribute__((ext_vector_type(4), aligned(1))) mask16;
  __shared__ int sums[16];
  const int b = blockIdx.x, M = a.M, lane = threadIdx.x & 63, w = threadIdx.x >> 6;
  const uint8_t* mask = a.mask + b * a.mask_b;
  const int len = a.lens ? min(max(a.lens[b], 0), M) : M;
  constexpr int kStep = kListThreads * kListKeys;
  auto bits_at = [&](int key) -> unsigned {      // which of 16 keys are seen
    unsigned bits = 0;
    if (key + kListKeys <= M) {
      const mask16 x = *reinterpret_cast<const mask16*>(mask + key);
#pragma unroll
      for (int e = 0; e < kListKeys; ++e) bits |= ((x[e / 4] >> (8 * (e % 4))) & 255u) != 0 ? 1u << e : 0u;
    } else {
      for (int e = 0; e < kListKeys; ++e)
        if (key + e < M && mask[key + e]) bits |= 1u << e;
    }
    const int left = len - key;
    return left >= kListKeys ? bits : left > 0 ? bits & ((1u << left) - 1u) : 0u;
  };
  // the sum over the workgroup of what each lane has, and what the lanes before it have
  auto scan = [&](int x, int& before) -> int {
    int run = x;
#pragma unroll
    for (int d = 1; d < 64; d *= 2) {
      const int y = __shfl_up(run, d);
      if (lane >= d) run += y;
    }
    __syncthreads();
    if (lane == 63) sums[w] = run;
    __syncthreads();
    int all = 0;
    before = run - x;
    for (int j = 0; j < kListThreads / 64; ++j) {
      if (j < w) before += sums[j];
      all += sums[j];
    }
    return all;
  };
  int mine = 0, before;
  for (int key = threadIdx.x * kListKeys; key < M; key += kStep) mine += __popc(bits_at(key));
  const int total = scan(mine, before);
  if (threadIdx.x == 0) a.seen[b] = total;
  int32_t* rows = a.rows + (int64_t)b * M;
  int done = 0;                                   // seen keys of earlier steps
  for (int first = 0; first < M; first += kStep) {
    const int key = first + threadIdx.x * kListKeys;
    const unsigned bits = key < M ? bits_at(key) : 0u;
    const int all = scan(__popc(bits), before);
    int seen = done + before, hidden = total + key - seen;
    for (int e = 0; e < kListKeys && key + e < M; ++e) {
      if (bits >> e & 1) rows[seen++] = key + e;
      else rows[hidden++] = key + e;
    }
    done += all;
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
  if (s.narrow) launch_qt<D, 1>(a, stream);
  else launch_qt<D, 2>(a, stream);
  if (a.splits == 1) return;
  if (a.lse) hipLaunchKernelGGL((cross_join_kernel<D, true>), dim3(a.B * a.Hkv * a.R), dim3(kThreads), 0, stream, a);
  else hipLaunchKernelGGL((cross_join_kernel<D, false>), dim3(a.B * a.Hkv * a.R), dim3(kThreads), 0, stream, a);
}

}  // namespace

static size_t up256(size_t x) { return (x + 255) / 256 * 256; }

CrossShape cross_shape(int B, int Hkv, int G, int N, int M, int D, bool mask) {
  CrossShape s{};
  const int64_t heads = (int64_t)B * Hkv, R = (int64_t)G * N;
  s.narrow = heads * ((R + 127) / 128) < 512;
  s.tiles = (int)((R + (s.narrow ? 63 : 127)) / (s.narrow ? 64 : 128));
  // keys are divided where the tiles are fewer than the card's places for workgroups
  const int64_t wgs = heads * s.tiles;
  int64_t splits = wgs < 512 ? 1024 / wgs : 1;
  if (splits > (M + 255) / 256) splits = (M + 255) / 256;
  s.splits = (int)(splits < 1 ? 1 : splits);
  size_t at = 0;
  if (mask) {
    s.rows_at = at;
    at += up256((size_t)B * M * 4);
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

hipError_t launch_cross_rows(const CrossArgs& a, hipStream_t stream) {
  hipLaunchKernelGGL(cross_rows_kernel, dim3(a.B), dim3(kListThreads), 0, stream, a);
  return hipGetLastError();
}

hipError_t launch_cross_attention(const CrossArgs& a, const CrossShape& s, hipStream_t stream) {
  if (a.mask) {
    const hipError_t e = launch_cross_rows(a, stream);
    if (e != hipSuccess) return e;
  }
  if (a.D == 64) launch_d<64>(a, s, stream);
  else if (a.D == 112) launch_d<112>(a, s, stream);
  else launch_d<128>(a, s, stream);
  return hipGetLastError();
}

}  // namespace sva
