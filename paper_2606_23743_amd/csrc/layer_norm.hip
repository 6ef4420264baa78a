// Layer norm of rows x[b, n, :] and its gradients:
//   xhat = (x - mean) rstd, rstd = 1 / sqrt(var + eps), y = xhat w + bias
//   dx = rstd (g - mean(g) - xhat mean(g xhat)), g = dy w
//   dw = sum of dy xhat, dbias = sum of dy, over all rows or an entry's
// with w = unit + weight (unit 1: a scale around one, as adaptive norms have it).
//
// Bound by HBM, and next to it by vector operations (an element is read and written once;
// 16 lanes a clock leave some twenty operations for it).  A row stays in registers from its
// load to its store, in pieces of eight elements.  Forward: 16 or 32 lanes or a wave hold a
// row of up to 6,144 channels, and no wave waits for another; longer ones a workgroup.
// Gradients: a wave up to 1,024, then a workgroup, whose lanes keep the sums of their
// columns for the weights' gradients in registers.  A workgroup takes rows of one batch
// entry, so the weights are loaded once; the next rows are on their way while one is worked
// on, and workgroups are a whole number per CU, each with as many rows.  Means are sums of
// differences or of the elements in a tree, corrected by the mean of the deviations or by the
// quotient's remainder; squares are of deviations from the mean, so no difference of large
// sums is ever taken.  The weights' gradients are written once per
// workgroup and added in a fixed order by a second launch: the same call gives the same bits.
//
// 63,240 x 4,096 bf16: 207 us (5.0 TB/s), gradients 286 (5.4); 65,520 x 2,240: 116 and 171;
// 23,403 x 1,001 float32: 43 and 60.  With a workgroup to every row and one row ahead the
// first took 237 and 358, the second 185 and 240.
#include <type_traits>

#include "norm_args.h"

namespace sva {
namespace {

typedef __attribute__((ext_vector_type(4))) unsigned u32x4;
typedef __attribute__((ext_vector_type(2))) float f32x2;
typedef __attribute__((ext_vector_type(2))) __bf16 bf16x2;
typedef u32x4 __attribute__((aligned(4))) u32x4a4;
typedef u32x4 __attribute__((aligned(2))) u32x4a2;

constexpr int E = 8;                          // elements of a piece

template <bool F32>
using Elem = std::conditional_t<F32, float, uint16_t>;

__device__ __forceinline__ float wide(uint16_t x) { return __uint_as_float((uint32_t)x << 16); }

// A piece as it lies in memory: eight bf16 or float32 elements.
template <bool F32>
struct Piece {
  uint32_t w[F32 ? 8 : 4];
};

template <bool F32, bool ALIGNED>
__device__ __forceinline__ Piece<F32> load_piece(const Elem<F32>* p) {
  using W = std::conditional_t<ALIGNED, u32x4, std::conditional_t<F32, u32x4a4, u32x4a2>>;
  Piece<F32> x;
#pragma unroll
  for (int i = 0; i < (F32 ? 2 : 1); ++i) {
    const u32x4 v = reinterpret_cast<const W*>(p)[i];
#pragma unroll
    for (int j = 0; j < 4; ++j) x.w[4 * i + j] = v[j];
  }
  return x;
}

// the first n of eight elements, zeros behind them
template <bool F32>
__device__ __forceinline__ Piece<F32> load_part(const Elem<F32>* p, int n) {
  Piece<F32> x{};
#pragma unroll
  for (int e = 0; e < E; ++e)
    if (e < n) {
      if constexpr (F32) x.w[e] = __float_as_uint(p[e]);
      else x.w[e / 2] |= (uint32_t)p[e] << (16 * (e & 1));
    }
  return x;
}

template <bool F32>
__device__ __forceinline__ void widen(const Piece<F32>& x, float (&y)[E]) {
#pragma unroll
  for (int e = 0; e < E; ++e) {
    if constexpr (F32) y[e] = __uint_as_float(x.w[e]);
    else y[e] = __uint_as_float(e & 1 ? x.w[e / 2] & 0xFFFF0000u : x.w[e / 2] << 16);
  }
}

template <bool F32>
__device__ __forceinline__ Piece<F32> narrow(const float (&y)[E]) {
  Piece<F32> x;
#pragma unroll
  for (int i = 0; i < (F32 ? 8 : 4); ++i) {
    if constexpr (F32) {
      x.w[i] = __float_as_uint(y[i]);
    } else {
      const f32x2 f = {y[2 * i], y[2 * i + 1]};
      x.w[i] = __builtin_bit_cast(uint32_t, __builtin_convertvector(f, bf16x2));
    }
  }
  return x;
}

template <bool F32, bool ALIGNED>
__device__ __forceinline__ void store_piece(Elem<F32>* p, const Piece<F32>& x, int n) {
  using W = std::conditional_t<ALIGNED, u32x4, std::conditional_t<F32, u32x4a4, u32x4a2>>;
  if (ALIGNED || n >= E) {
#pragma unroll
    for (int i = 0; i < (F32 ? 2 : 1); ++i) {
      u32x4 v;
#pragma unroll
      for (int j = 0; j < 4; ++j) v[j] = x.w[4 * i + j];
      reinterpret_cast<W*>(p)[i] = v;
    }
  } else {
#pragma unroll
    for (int e = 0; e < E; ++e)
      if (e < n) {
        if constexpr (F32) p[e] = __uint_as_float(x.w[e]);
        else p[e] = (uint16_t)(x.w[e / 2] >> (16 * (e & 1)));
      }
  }
}

template <int CTRL>
__device__ __forceinline__ float dpp_add(float x) {
  return x + __int_as_float(__builtin_amdgcn_update_dpp(0, __float_as_int(x), CTRL, 0xf, 0xf, true));
}

// the sum over 16, 32 or 64 neighbouring lanes, the same bits in each of them
template <int L>
__device__ __forceinline__ float lanes_sum(float x) {
  x = dpp_add<0xB1>(x);                       // lane ^ 1
  x = dpp_add<0x4E>(x);                       // lane ^ 2
  x = dpp_add<0x141>(x);                      // mirrored in eight lanes
  x = dpp_add<0x140>(x);                      // mirrored in sixteen
  if constexpr (L >= 32) {
    const auto r = __builtin_amdgcn_permlane16_swap(__float_as_uint(x), __float_as_uint(x), false, false);
    x = __uint_as_float(r[0]) + __uint_as_float(r[1]);
  }
  if constexpr (L >= 64) {
    const auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
    x = __uint_as_float(r[0]) + __uint_as_float(r[1]);
  }
  return x;
}

// weight c as float32: `none` where there are no weights or no channel c
__device__ __forceinline__ float weight_at(const void* w, bool bf16, int64_t at, float none, float add, int c, int C) {
  if (!w || c >= C) return none;
  return add + (bf16 ? wide(static_cast<const uint16_t*>(w)[at + c]) : static_cast<const float*>(w)[at + c]);
}

// The weights of a lane's pieces as float32 (ones plus the offset where there are none).
template <int V>
__device__ __forceinline__ void load_weights(const void* w, bool bf16, int64_t at, float none, float add, int lane0, int step,
                                             int C, float (&out)[V][E]) {
#pragma unroll
  for (int v = 0; v < V; ++v)
#pragma unroll
    for (int e = 0; e < E; ++e) out[v][e] = weight_at(w, bf16, at, none, add, (lane0 + v * step) * E + e, C);
}

// How a launch's lanes take rows.  L lanes hold a row (L = 0: the workgroup), V pieces
// a lane; piece v of lane i of the row is number i + v * step.
template <int L>
struct Place {
  int step, lane, group, groups;              // lanes of a row, this lane among them, its row among the workgroup's
  __device__ Place() {
    step = L ? L : (int)blockDim.x;
    lane = L ? threadIdx.x % (L ? L : 1) : threadIdx.x;
    group = L ? threadIdx.x / (L ? L : 1) : 0;
    groups = L ? kNormThreads / (L ? L : 1) : 1;
  }
};

template <bool F32, bool ALIGNED, int V>
__device__ __forceinline__ void load_row(const Elem<F32>* row, int lane, int step, int C, Piece<F32> (&x)[V]) {
#pragma unroll
  for (int v = 0; v < V; ++v) {
    const int c = (lane + v * step) * E;
    if (c + E <= C) x[v] = load_piece<F32, ALIGNED>(row + c);
    else if (!ALIGNED && c < C) x[v] = load_part<F32>(row + c, C - c);
    else x[v] = Piece<F32>{};
  }
}

// a tree of eight
__device__ __forceinline__ float sum8(const float (&f)[E]) {
  return ((f[0] + f[1]) + (f[2] + f[3])) + ((f[4] + f[5]) + (f[6] + f[7]));
}

// Rows of up to 6,144 channels: L lanes of a wave hold one, V pieces a lane, and no wave
// waits for another.  Vector operations bound it as much as HBM does (16 lanes a clock,
// some seven operations an element), so the row's deviations stay in registers, and the
// weights of longer rows, which would crowd them out, lie in LDS.
template <bool F32, bool ALIGNED, int L, int V>
__global__ __launch_bounds__(kNormThreads) void norm_wave_kernel(NormArgs a) {
  constexpr int PF = V <= 2 ? 4 : V <= 4 ? 2 : 1;  // rows on their way
  constexpr bool IN_LDS = V > 1;
  __shared__ float4 lds_w[IN_LDS ? 2 * V * 2 * 64 : 1];
  const int C = a.C, b = blockIdx.x / a.parts, part = blockIdx.x - b * a.parts;
  const int lane = threadIdx.x % L;
  const Elem<F32>* xs = static_cast<const Elem<F32>*>(a.x.p) + b * a.x.sb;
  Elem<F32>* ys = static_cast<Elem<F32>*>(a.y.p) + b * a.y.sb;
  const int stride = a.parts * (kNormThreads / L);
  int n = part * (kNormThreads / L) + threadIdx.x / L;

  Piece<F32> ring[PF][V];
#pragma unroll
  for (int u = 0; u < PF; ++u)
    if (n + (int64_t)u * stride < a.N) load_row<F32, ALIGNED, V>(xs + (n + (int64_t)u * stride) * a.x.sn, lane, L, C, ring[u]);

  float w[IN_LDS ? 1 : V][E], bias[IN_LDS ? 1 : V][E];
  if constexpr (IN_LDS) {
    // as halves of pieces, each in the order of the lanes: no two of them on one bank
    for (int i = threadIdx.x; i < V * 2 * 64; i += kNormThreads) {
      const int c = (i / 128 * 64 + i % 64) * E + i / 64 % 2 * 4;
      float q[2][4];
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        q[0][e] = weight_at(a.w, a.w_bf16, b * a.w_b, 1.0f, a.unit, c + e, C);
        q[1][e] = weight_at(a.bias, a.w_bf16, b * a.bias_b, 0.0f, 0.0f, c + e, C);
      }
      lds_w[i] = make_float4(q[0][0], q[0][1], q[0][2], q[0][3]);
      lds_w[V * 2 * 64 + i] = make_float4(q[1][0], q[1][1], q[1][2], q[1][3]);
    }
    __syncthreads();
  } else {
    load_weights<V>(a.w, a.w_bf16, b * a.w_b, 1.0f, a.unit, lane, L, C, w);
    load_weights<V>(a.bias, a.w_bf16, b * a.bias_b, 0.0f, 0.0f, lane, L, C, bias);
  }
  const float inv_c = 1.0f / (float)C;

  // zeros behind the row's end, in the one piece of its lanes that may hold it
  auto clear_tail = [&](float (&f)[E], int v) {
    if (ALIGNED || (v + 1) * L * E <= C) return;
    int left = C - (lane + v * L) * E;
    asm volatile("" : "+v"(left));             // (not eight masks kept from row to row)
#pragma unroll
    for (int e = 0; e < E; ++e) f[e] = e < left ? f[e] : 0.0f;
  };
  auto row = [&](Piece<F32> (&x)[V]) {
    // The sum of a float32 row is of differences from its first element: a mean far from zero
    // then costs it no digits (sums of bf16 elements as alike as that are exact).  Where the first
    // is far from the others the differences have lost theirs, so deviations are of the row
    // itself, and what their sum leaves is the mean's error, which they and the mean are rid of:
    // rows of 4,096 whose first channel is 1e5 had lost up to 0.4 % of a deviation in every other.
    float f[V][E], sum = 0.0f, first = 0.0f;
    if constexpr (F32) first = __shfl(__uint_as_float(x[0].w[0]), 0, L);
#pragma unroll
    for (int v = 0; v < V; ++v) {
      const int c = (lane + v * L) * E;
      widen<F32>(x[v], f[v]);
      if (c < C) {
        if constexpr (F32) {
          float d[E];
#pragma unroll
          for (int e = 0; e < E; ++e) d[e] = f[v][e] - first;
          clear_tail(d, v);
          sum += sum8(d);
        } else {
          sum += sum8(f[v]);
        }
      }
    }
    sum = lanes_sum<L>(sum);
    float mean = first + sum * inv_c, more = 0.0f, m2 = 0.0f;
    if constexpr (F32) {
      float dev = 0.0f;
#pragma unroll
      for (int v = 0; v < V; ++v)
        if ((lane + v * L) * E < C) {
#pragma unroll
          for (int e = 0; e < E; ++e) f[v][e] -= mean;
          clear_tail(f[v], v);
          dev += sum8(f[v]);
        }
      more = lanes_sum<L>(dev) * inv_c;
    } else {
      // The sum of equal bf16 elements is exact, times 1 / C it may be a step off them; with the
      // remainder's share it is their value (the correction above: 23.6 -> 24.8 us for
      // 30,000 x 1,024; this: no difference).
      mean = fmaf(fmaf(-mean, (float)C, sum), inv_c, mean);
    }
    const float off = F32 ? more : mean;
    mean += more;
#pragma unroll
    for (int v = 0; v < V; ++v) {
      const int c = (lane + v * L) * E;
      if (c < C) {
#pragma unroll
        for (int e = 0; e < E; ++e) f[v][e] -= off;
        clear_tail(f[v], v);
#pragma unroll
        for (int e = 0; e < E; ++e) m2 = fmaf(f[v][e], f[v][e], m2);
      }
    }
    const float rstd = 1.0f / sqrtf(lanes_sum<L>(m2) * inv_c + a.eps);
    if (lane == 0) {
      if (a.mean) a.mean[(int64_t)b * a.N + n] = mean;
      if (a.rstd) a.rstd[(int64_t)b * a.N + n] = rstd;
    }
    Elem<F32>* y = ys + n * a.y.sn;
#pragma unroll
    for (int v = 0; v < V; ++v) {
      const int c = (lane + v * L) * E;
      if (c < C) {
#pragma unroll
        for (int h = 0; h < 2; ++h) {
          float wq[4], bq[4];
          if constexpr (IN_LDS) {
            const float4 p = lds_w[(v * 2 + h) * 64 + lane], q = lds_w[V * 2 * 64 + (v * 2 + h) * 64 + lane];
            wq[0] = p.x, wq[1] = p.y, wq[2] = p.z, wq[3] = p.w;
            bq[0] = q.x, bq[1] = q.y, bq[2] = q.z, bq[3] = q.w;
          } else {
#pragma unroll
            for (int e = 0; e < 4; ++e) {
              wq[e] = w[v][4 * h + e];
              bq[e] = bias[v][4 * h + e];
            }
          }
#pragma unroll
          for (int e = 0; e < 4; ++e) f[v][4 * h + e] = fmaf(f[v][4 * h + e] * rstd, wq[e], bq[e]);
        }
        store_piece<F32, ALIGNED>(y + c, narrow<F32>(f[v]), C - c);
      }
    }
    const int64_t later = n + (int64_t)PF * stride;
    if (later < a.N) load_row<F32, ALIGNED, V>(xs + later * a.x.sn, lane, L, C, x);
    n += stride;
  };
  while (n < a.N) {
#pragma unroll
    for (int u = 0; u < PF; ++u)
      if (n < a.N) row(ring[u]);
  }
}

// Longer rows: a workgroup holds one.  A wave forms mean and squared deviations of its own
// part; the waves' parts are joined as (count, mean, M2), one barrier a row.
template <bool F32, bool ALIGNED, int V, int T>
__global__ __launch_bounds__(T) void norm_kernel(NormArgs a) {
  constexpr int PF = T > 512 ? 1 : 2;
  const Place<0> at;
  const int C = a.C, b = blockIdx.x / a.parts, part = blockIdx.x - b * a.parts;
  __shared__ float2 joined[2][16];            // (mean, M2) of the waves' parts, two rows in turn

  float w[V][E], bias[V][E];
  load_weights<V>(a.w, a.w_bf16, b * a.w_b, 1.0f, a.unit, at.lane, at.step, C, w);
  load_weights<V>(a.bias, a.w_bf16, b * a.bias_b, 0.0f, 0.0f, at.lane, at.step, C, bias);
  const Elem<F32>* xs = static_cast<const Elem<F32>*>(a.x.p) + b * a.x.sb;
  Elem<F32>* ys = static_cast<Elem<F32>*>(a.y.p) + b * a.y.sb;

  const int waves = blockDim.x / 64, wave = threadIdx.x / 64;
  int mine = 0;                               // elements that this wave holds
  for (int v = 0; v < V; ++v) mine += min(max(C - (v * at.step + wave * 64) * E, 0), 64 * E);
  const float inv_c = 1.0f / (float)C, inv_mine = mine ? 1.0f / (float)mine : 0.0f;

  // A row's loads go out PF rows ahead of its use: one row ahead left HBM waiting
  Piece<F32> ring[PF][V];
  const int stride = a.parts * at.groups;
  int n = part * at.groups + at.group, turn = 0;
#pragma unroll
  for (int u = 0; u < PF; ++u)
    if (n + (int64_t)u * stride < a.N) load_row<F32, ALIGNED, V>(xs + (n + (int64_t)u * stride) * a.x.sn, at.lane, at.step, C, ring[u]);
  // (a workgroup's lanes are at the same row)
  auto row = [&](Piece<F32> (&x)[V]) {
    float sum = 0.0f;
#pragma unroll
    for (int v = 0; v < V; ++v) {
      float f[E];
      widen<F32>(x[v], f);
#pragma unroll
      for (int e = 0; e < E; ++e) sum += f[e];
    }
    float mean = lanes_sum<64>(sum) * inv_mine, m2 = 0.0f, dev = 0.0f;
#pragma unroll
    for (int v = 0; v < V; ++v) {
      float f[E];
      widen<F32>(x[v], f);
#pragma unroll
      for (int e = 0; e < E; ++e) {
        const float d = (at.lane + v * at.step) * E + e < C ? f[e] - mean : 0.0f;
        dev += d;
        m2 = fmaf(d, d, m2);
      }
    }
    // what rounding left of the mean: the deviations' own
    dev = lanes_sum<64>(dev);
    m2 = lanes_sum<64>(m2);
    const float more = dev * inv_mine;
    mean += more;
    m2 = fmaxf(m2 - dev * more, 0.0f);
    if (threadIdx.x % 64 == 0) joined[turn][wave] = make_float2(mean, m2);
    __syncthreads();
    // the mean of the waves' means around the first one's, then their squares around it
    const float m0 = joined[turn][0].x;
    float off = 0.0f;
    for (int i = 0; i < waves; ++i) {
      int count = 0;
      for (int v = 0; v < V; ++v) count += min(max(C - (v * at.step + i * 64) * E, 0), 64 * E);
      off = fmaf((float)count, joined[turn][i].x - m0, off);
    }
    mean = m0 + off * inv_c;
    m2 = 0.0f;
    for (int i = 0; i < waves; ++i) {
      int count = 0;
      for (int v = 0; v < V; ++v) count += min(max(C - (v * at.step + i * 64) * E, 0), 64 * E);
      const float d = joined[turn][i].x - mean;
      m2 += joined[turn][i].y + (float)count * d * d;
    }
    const float rstd = 1.0f / sqrtf(m2 * inv_c + a.eps);
    if (at.lane == 0) {
      if (a.mean) a.mean[(int64_t)b * a.N + n] = mean;
      if (a.rstd) a.rstd[(int64_t)b * a.N + n] = rstd;
    }
    Elem<F32>* y = ys + n * a.y.sn;
#pragma unroll
    for (int v = 0; v < V; ++v) {
      const int c = (at.lane + v * at.step) * E;
      if (c < C) {
        float f[E];
        widen<F32>(x[v], f);
#pragma unroll
        for (int e = 0; e < E; ++e) f[e] = fmaf((f[e] - mean) * rstd, w[v][e], bias[v][e]);
        store_piece<F32, ALIGNED>(y + c, narrow<F32>(f), C - c);
      }
    }
    const int64_t later = n + (int64_t)PF * stride;
    if (later < a.N) load_row<F32, ALIGNED, V>(xs + later * a.x.sn, at.lane, at.step, C, x);
    n += stride;
    turn ^= 1;
  };
  while (n < a.N) {
#pragma unroll
    for (int u = 0; u < PF; ++u)
      if (n < a.N) row(ring[u]);
  }
}

template <bool F32, bool ALIGNED, int L, int V, int T, int R>
__global__ __launch_bounds__(T) void norm_grad_kernel(NormArgs a) {
  constexpr int PF = T > 512 ? 1 : R == 2 ? 2 : F32 ? 2 : 3;   // times R rows on their way
  const Place<L> at;
  const int C = a.C, b = blockIdx.x / a.parts, part = blockIdx.x - b * a.parts;
  __shared__ float2 joined[2][R][16];

  float w[V][E], dw[V][E] = {}, db[V][E] = {};
  load_weights<V>(a.w, a.w_bf16, b * a.w_b, 1.0f, a.unit, at.lane, at.step, C, w);
  const Elem<F32>* xs = static_cast<const Elem<F32>*>(a.x.p) + b * a.x.sb;
  const Elem<F32>* gs = static_cast<const Elem<F32>*>(a.dy.p) + b * a.dy.sb;
  Elem<F32>* outs = static_cast<Elem<F32>*>(a.y.p) + b * a.y.sb;
  const float* means = a.mean + (int64_t)b * a.N;
  const float* rstds = a.rstd + (int64_t)b * a.N;
  const int waves = blockDim.x / 64, wave = threadIdx.x / 64;
  const float inv_c = 1.0f / (float)C;

  struct Row {
    Piece<F32> x[V], g[V];
    float mean, rstd;
  };
  Row ring[PF][R];
  const int stride = a.parts * at.groups;
  int n = part * at.groups + at.group, turn = 0;
  // R rows a stride apart; one that is not there is zeros, and adds nothing
  auto load = [&](int64_t n, Row (&r)[R]) {
#pragma unroll
    for (int k = 0; k < R; ++k) {
      const int64_t m = n + (int64_t)k * stride;
      if (m < a.N) {
        load_row<F32, ALIGNED, V>(xs + m * a.x.sn, at.lane, at.step, C, r[k].x);
        load_row<F32, ALIGNED, V>(gs + m * a.dy.sn, at.lane, at.step, C, r[k].g);
        r[k].mean = means[m];
        r[k].rstd = rstds[m];
      } else {
        r[k] = Row{};
      }
    }
  };
  auto rows = [&](Row (&r)[R]) {
    float s1[R], s2[R], f[R][V][E], d[R][V][E];
#pragma unroll
    for (int k = 0; k < R; ++k) {
      s1[k] = s2[k] = 0.0f;
#pragma unroll
      for (int v = 0; v < V; ++v) {
        widen<F32>(r[k].x[v], f[k][v]);
        widen<F32>(r[k].g[v], d[k][v]);
        // Past the row's end x and dy are zero; so is xhat there, as a mean times rstd may be
        // infinite where no element of the row is far from it.
        int left = C - (at.lane + v * at.step) * E;
        const float mean = ALIGNED && left <= 0 ? 0.0f : r[k].mean;
#pragma unroll
        for (int e = 0; e < E; ++e) f[k][v][e] = (f[k][v][e] - mean) * r[k].rstd;       // xhat
        if (!ALIGNED && (v + 1) * at.step * E > C) {
          asm volatile("" : "+v"(left));       // (not eight masks kept from row to row)
#pragma unroll
          for (int e = 0; e < E; ++e) f[k][v][e] = e < left ? f[k][v][e] : 0.0f;
        }
#pragma unroll
        for (int e = 0; e < E; ++e) {
          dw[v][e] = fmaf(d[k][v][e], f[k][v][e], dw[v][e]);
          db[v][e] += d[k][v][e];
          d[k][v][e] *= w[v][e];                                   // g
          s1[k] += d[k][v][e];
          s2[k] = fmaf(d[k][v][e], f[k][v][e], s2[k]);
        }
      }
      s1[k] = lanes_sum<L ? L : 64>(s1[k]);
      s2[k] = lanes_sum<L ? L : 64>(s2[k]);
    }
    if constexpr (L == 0) {
      if (threadIdx.x % 64 == 0) {
#pragma unroll
        for (int k = 0; k < R; ++k) joined[turn][k][wave] = make_float2(s1[k], s2[k]);
      }
      __syncthreads();
#pragma unroll
      for (int k = 0; k < R; ++k) {
        s1[k] = s2[k] = 0.0f;
        for (int i = 0; i < waves; ++i) {
          s1[k] += joined[turn][k][i].x;
          s2[k] += joined[turn][k][i].y;
        }
      }
    }
#pragma unroll
    for (int k = 0; k < R; ++k) {
      const int64_t m = n + (int64_t)k * stride;
      if (m >= a.N) continue;
      const float m1 = s1[k] * inv_c, m2 = s2[k] * inv_c;
      Elem<F32>* out = outs + m * a.y.sn;
#pragma unroll
      for (int v = 0; v < V; ++v) {
        const int c = (at.lane + v * at.step) * E;
        if (c < C) {
#pragma unroll
          for (int e = 0; e < E; ++e) f[k][v][e] = r[k].rstd * ((d[k][v][e] - m1) - f[k][v][e] * m2);
          store_piece<F32, ALIGNED>(out + c, narrow<F32>(f[k][v]), C - c);
        }
      }
    }
    load(n + (int64_t)PF * R * stride, r);
    n += R * stride;
    turn ^= 1;
  };
#pragma unroll
  for (int u = 0; u < PF; ++u) load(n + (int64_t)u * R * stride, ring[u]);
  while (n < a.N) {
#pragma unroll
    for (int u = 0; u < PF; ++u)
      if (n < a.N) rows(ring[u]);
  }
  if (!a.dw && !a.db) return;
  // an entry's only workgroup has its sums whole
  float* to_w = a.partial ? a.partial + (int64_t)blockIdx.x * 2 * C : a.dw ? a.dw + (int64_t)b * C : nullptr;
  float* to_b = a.partial ? to_w + C : a.db ? a.db + (int64_t)b * C : nullptr;
  if constexpr (L == 0) {
#pragma unroll
    for (int v = 0; v < V; ++v)
#pragma unroll
      for (int e = 0; e < E; ++e) {
        const int c = (at.lane + v * at.step) * E + e;
        if (c < C) {
          if (to_w) to_w[c] = dw[v][e];
          if (to_b) to_b[c] = db[v][e];
        }
      }
  } else {
    // the workgroup's rows of lanes are added in their order
    __shared__ float both[L ? 2 * kNormThreads * V * E : 1];
    constexpr int kRow = 2 * (L ? L : 1) * V * E;
#pragma unroll
    for (int v = 0; v < V; ++v)
#pragma unroll
      for (int e = 0; e < E; ++e) {
        const int c = (at.lane + v * at.step) * E + e;
        both[at.group * kRow + c] = dw[v][e];
        both[at.group * kRow + kRow / 2 + c] = db[v][e];
      }
    __syncthreads();
    for (int c = threadIdx.x; c < 2 * C; c += kNormThreads) {
      const int col = c < C ? c : kRow / 2 + c - C;
      float s = 0.0f;
      for (int i = 0; i < at.groups; ++i) s += both[i * kRow + col];
      float* to = c < C ? to_w : to_b;
      if (to) to[c < C ? c : c - C] = s;
    }
  }
}

// Sums the workgroups' parts of the weights' gradients: partial [entries][parts][2][C]
// -> dw, db [entries][C].  64 columns a workgroup, 16 runs of parts, then those in order.
__global__ __launch_bounds__(1024) void norm_join_kernel(const float* partial, float* dw, float* db, int C, int parts) {
  __shared__ float runs[16][64];
  const int col = blockIdx.x * 64 + (threadIdx.x & 63), run = threadIdx.x >> 6;
  const int64_t entry = blockIdx.y;
  const float* from = partial + entry * parts * 2 * C;
  float s = 0.0f;
  if (col < 2 * C) {
    const int first = (int)((int64_t)parts * run / 16), last = (int)((int64_t)parts * (run + 1) / 16);
#pragma unroll 8
    for (int i = first; i < last; ++i) s += from[(int64_t)i * 2 * C + col];
  }
  runs[run][threadIdx.x & 63] = s;
  __syncthreads();
  if (run == 0 && col < 2 * C) {
    s = 0.0f;
#pragma unroll
    for (int i = 0; i < 16; ++i) s += runs[i][threadIdx.x];
    float* to = col < C ? dw : db;
    if (to) to[entry * C + (col < C ? col : col - C)] = s;
  }
}

template <bool F32, bool ALIGNED>
void launch_as(const NormArgs& a, const NormShape& s, bool grad, hipStream_t stream) {
  using std::integral_constant;
  auto go = [&](auto kernel) { hipLaunchKernelGGL(kernel, dim3(a.B * a.parts), dim3(s.threads), 0, stream, a); };
  if (grad) {
    if (s.lanes == 16) go(norm_grad_kernel<F32, ALIGNED, 16, 1, kNormThreads, 1>);
    else if (s.lanes == 32) go(norm_grad_kernel<F32, ALIGNED, 32, 1, kNormThreads, 1>);
    else if (s.lanes == 64 && s.pieces == 1) go(norm_grad_kernel<F32, ALIGNED, 64, 1, kNormThreads, 1>);
    else if (s.lanes == 64) go(norm_grad_kernel<F32, ALIGNED, 64, 2, kNormThreads, 1>);
    else if (s.pieces == 1) go(norm_grad_kernel<F32, ALIGNED, 0, 1, 512, 2>);
    else if (s.threads <= 512) go(norm_grad_kernel<F32, ALIGNED, 0, 2, 512, 1>);
    else go(norm_grad_kernel<F32, ALIGNED, 0, 2, 1024, 1>);
  } else if (s.lanes) {
    if (s.lanes == 16) go(norm_wave_kernel<F32, ALIGNED, 16, 1>);
    else if (s.lanes == 32) go(norm_wave_kernel<F32, ALIGNED, 32, 1>);
    else if (s.pieces == 1) go(norm_wave_kernel<F32, ALIGNED, 64, 1>);
    else if (s.pieces == 2) go(norm_wave_kernel<F32, ALIGNED, 64, 2>);
    else if (s.pieces == 4) go(norm_wave_kernel<F32, ALIGNED, 64, 4>);
    else if (s.pieces == 8) go(norm_wave_kernel<F32, ALIGNED, 64, 8>);
    else go(norm_wave_kernel<F32, ALIGNED, 64, 12>);
  } else {
    if (s.threads <= 512) go(norm_kernel<F32, ALIGNED, 2, 512>);
    else go(norm_kernel<F32, ALIGNED, 2, 1024>);
  }
}

hipError_t launch(const NormArgs& a, const NormShape& s, bool grad, hipStream_t stream) {
  if (a.f32) {
    if (a.aligned) launch_as<true, true>(a, s, grad, stream);
    else launch_as<true, false>(a, s, grad, stream);
  } else {
    if (a.aligned) launch_as<false, true>(a, s, grad, stream);
    else launch_as<false, false>(a, s, grad, stream);
  }
  return hipGetLastError();
}

}  // namespace

// A row belongs to 16 or 32 lanes or a wave as long as a wave's registers hold it, which in the
// gradients, that keep the sums of their columns too, is up to 1,024 channels (23,403 x 1,001
// float32: 60 us, by a workgroup 72), forward up to 6,144 (63,240 x 4,096: 204 us, by a workgroup
// 237).  Workgroups are as many as a CU's registers take in whole rounds: gradients of 65,520 x
// 2,240 with 704 threads a CU 171 us, 1,024 215, 1,600 209.  Up to 384 pieces a lane holds
// one, more need two: a gradient's workgroup of 512 lanes with one piece each takes 313 us
// for 63,240 x 4,096, of 256 with two 288.
NormShape norm_shape(int B, int N, int C, bool grad, bool per_entry) {
  NormShape s{};
  const int pieces = (C + E - 1) / E;
  int per_cu;                                   // workgroups of a CU, a whole number: each takes as many rows
  s.threads = kNormThreads;
  if (pieces <= 64) {
    s.lanes = pieces <= 16 ? 16 : pieces <= 32 ? 32 : 64;
    s.pieces = 1;
    per_cu = grad ? 3 : 6;
  } else if (grad && pieces <= 2 * 64) {
    s.lanes = 64;
    s.pieces = 2;
    per_cu = 3;
  } else if (!grad && pieces <= 12 * 64) {
    s.lanes = 64;
    s.pieces = pieces <= 2 * 64 ? 2 : pieces <= 4 * 64 ? 4 : pieces <= 8 * 64 ? 8 : 12;
    per_cu = s.pieces == 2 ? 6 : s.pieces == 4 ? 4 : s.pieces == 8 ? 3 : 2;
  } else {
    s.pieces = pieces <= 384 ? 1 : 2;
    s.threads = ((pieces + s.pieces - 1) / s.pieces + 63) / 64 * 64;
    per_cu = (grad ? 704 : 2048) / s.threads;
    if (per_cu < 1) per_cu = 1;
  }
  const int rows = s.lanes ? kNormThreads / s.lanes : 1;     // of a workgroup at a time
  int64_t parts = (256 * per_cu + B - 1) / B;
  const int64_t most = ((int64_t)N + rows - 1) / rows;
  if (parts > most) parts = most;
  s.parts = (int)parts;
  s.ws_bytes = grad && !(per_entry && s.parts == 1) ? (size_t)B * s.parts * 2 * C * sizeof(float) : 0;
  return s;
}

hipError_t launch_layer_norm(const NormArgs& a, const NormShape& s, hipStream_t stream) { return launch(a, s, false, stream); }

hipError_t launch_layer_norm_grad(const NormArgs& a, const NormShape& s, int entries, hipStream_t stream) {
  hipError_t e = launch(a, s, true, stream);
  if (e != hipSuccess || !a.partial) return e;
  hipLaunchKernelGGL(norm_join_kernel, dim3((2 * a.C + 63) / 64, entries), dim3(1024), 0, stream, a.partial, a.dw, a.db, a.C,
                     (int)((int64_t)a.B * a.parts / entries));
  return hipGetLastError();
}

}  // namespace sva
