// Layer norm of rows x[b, n, :] and its gradients:
//   xhat = (x - mean) rstd, rstd = 1 / sqrt(var + eps), y = xhat w + bias
//   dx = rstd (g - mean(g) - xhat mean(g xhat)), g = dy w
//   dw = sum of dy xhat, dbias = sum of dy, over all rows or an entry's
// with w = unit + weight (unit 1: a scale around one, as adaptive norms have it).
//
// Bound by HBM: an element is read (x; dy) and written once and costs some ten
// operations.  A row stays in registers from its load to its store, in pieces of
// eight elements: 16 or 32 lanes or a wave hold a short row, a whole workgroup a
// longer one, V pieces a lane.  A workgroup takes rows of one batch entry, so the
// weights are loaded once, and while it reduces a row the next one is on its way.
// A wave forms mean and squared deviations of its own part by two sums over its
// lanes; the waves' parts are joined as (count, mean, M2), one barrier a row, so
// no difference of large sums is ever taken.  The weights' gradients are summed
// over a workgroup's rows in registers, written once per workgroup and added in a
// fixed order by a second launch: the same call gives the same bits.
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

// The weights of a lane's pieces as float32 (ones plus the offset where there are none).
template <int V>
__device__ __forceinline__ void load_weights(const void* w, bool bf16, int64_t at, float none, float add, int lane0, int step,
                                             int C, float (&out)[V][E]) {
#pragma unroll
  for (int v = 0; v < V; ++v)
#pragma unroll
    for (int e = 0; e < E; ++e) {
      const int c = (lane0 + v * step) * E + e;
      out[v][e] = none;
      if (w && c < C) out[v][e] = add + (bf16 ? wide(static_cast<const uint16_t*>(w)[at + c]) : static_cast<const float*>(w)[at + c]);
    }
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

template <bool F32, bool ALIGNED, int L, int V, int T>
__global__ __launch_bounds__(T) void norm_kernel(NormArgs a) {
  const Place<L> at;
  const int C = a.C, b = blockIdx.x / a.parts, part = blockIdx.x - b * a.parts;
  __shared__ float2 joined[2][16];            // (mean, M2) of the waves' parts, two rows in turn

  float w[V][E], bias[V][E];
  load_weights<V>(a.w, a.w_bf16, b * a.w_b, 1.0f, a.unit, at.lane, at.step, C, w);
  load_weights<V>(a.bias, a.w_bf16, b * a.bias_b, 0.0f, 0.0f, at.lane, at.step, C, bias);
  const Elem<F32>* xs = static_cast<const Elem<F32>*>(a.x.p) + b * a.x.sb;
  Elem<F32>* ys = static_cast<Elem<F32>*>(a.y.p) + b * a.y.sb;

  // elements of this lane's part: the wave's own where a workgroup holds the row
  const int waves = blockDim.x / 64, wave = threadIdx.x / 64;
  int mine = 0;                               // elements that this wave (L lanes) holds
  if (L) {
    mine = C;
  } else {
    for (int v = 0; v < V; ++v) mine += min(max(C - (v * at.step + wave * 64) * E, 0), 64 * E);
  }
  const float inv_c = 1.0f / (float)C, inv_mine = mine ? 1.0f / (float)mine : 0.0f;

  Piece<F32> x[V], next[V];
  const int stride = a.parts * at.groups;
  int n = part * at.groups + at.group, turn = 0;
  if (n < a.N) load_row<F32, ALIGNED, V>(xs + n * a.x.sn, at.lane, at.step, C, x);
  // (a workgroup's lanes are at the same row, or there is no barrier below)
  for (; n < a.N; n += stride, turn ^= 1) {
    if (n + stride < a.N) load_row<F32, ALIGNED, V>(xs + (n + stride) * a.x.sn, at.lane, at.step, C, next);
    float sum = 0.0f;
#pragma unroll
    for (int v = 0; v < V; ++v) {
      float f[E];
      widen<F32>(x[v], f);
#pragma unroll
      for (int e = 0; e < E; ++e) sum += f[e];
    }
    float mean = lanes_sum<L ? L : 64>(sum) * inv_mine, m2 = 0.0f, dev = 0.0f;
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
    dev = lanes_sum<L ? L : 64>(dev);
    m2 = lanes_sum<L ? L : 64>(m2);
    const float more = dev * inv_mine;
    mean += more;
    m2 = fmaxf(m2 - dev * more, 0.0f);
    if constexpr (L == 0) {
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
      x[v] = next[v];
    }
  }
}

template <bool F32, bool ALIGNED, int L, int V, int T>
__global__ __launch_bounds__(T) void norm_grad_kernel(NormArgs a) {
  const Place<L> at;
  const int C = a.C, b = blockIdx.x / a.parts, part = blockIdx.x - b * a.parts;
  __shared__ float2 joined[2][16];

  float w[V][E], dw[V][E] = {}, db[V][E] = {};
  load_weights<V>(a.w, a.w_bf16, b * a.w_b, 1.0f, a.unit, at.lane, at.step, C, w);
  const Elem<F32>* xs = static_cast<const Elem<F32>*>(a.x.p) + b * a.x.sb;
  const Elem<F32>* gs = static_cast<const Elem<F32>*>(a.dy.p) + b * a.dy.sb;
  Elem<F32>* outs = static_cast<Elem<F32>*>(a.y.p) + b * a.y.sb;
  const float* means = a.mean + (int64_t)b * a.N;
  const float* rstds = a.rstd + (int64_t)b * a.N;
  const int waves = blockDim.x / 64, wave = threadIdx.x / 64;
  const float inv_c = 1.0f / (float)C;

  Piece<F32> x[V], g[V], xn[V], gn[V];
  float mean = 0.0f, rstd = 0.0f, mean_n = 0.0f, rstd_n = 0.0f;
  const int stride = a.parts * at.groups;
  int n = part * at.groups + at.group, turn = 0;
  if (n < a.N) {
    load_row<F32, ALIGNED, V>(xs + n * a.x.sn, at.lane, at.step, C, x);
    load_row<F32, ALIGNED, V>(gs + n * a.dy.sn, at.lane, at.step, C, g);
    mean = means[n];
    rstd = rstds[n];
  }
  for (; n < a.N; n += stride, turn ^= 1) {
    if (n + stride < a.N) {
      load_row<F32, ALIGNED, V>(xs + (n + stride) * a.x.sn, at.lane, at.step, C, xn);
      load_row<F32, ALIGNED, V>(gs + (n + stride) * a.dy.sn, at.lane, at.step, C, gn);
      mean_n = means[n + stride];
      rstd_n = rstds[n + stride];
    }
    float s1 = 0.0f, s2 = 0.0f;
#pragma unroll
    for (int v = 0; v < V; ++v) {
      float f[E], d[E];
      widen<F32>(x[v], f);
      widen<F32>(g[v], d);
#pragma unroll
      for (int e = 0; e < E; ++e) {
        // past the row's end dy is zero, and so are all four
        const float xh = (f[e] - mean) * rstd, gw = d[e] * w[v][e];
        dw[v][e] = fmaf(d[e], xh, dw[v][e]);
        db[v][e] += d[e];
        s1 += gw;
        s2 = fmaf(gw, xh, s2);
      }
    }
    s1 = lanes_sum<L ? L : 64>(s1);
    s2 = lanes_sum<L ? L : 64>(s2);
    if constexpr (L == 0) {
      if (threadIdx.x % 64 == 0) joined[turn][wave] = make_float2(s1, s2);
      __syncthreads();
      s1 = s2 = 0.0f;
      for (int i = 0; i < waves; ++i) {
        s1 += joined[turn][i].x;
        s2 += joined[turn][i].y;
      }
    }
    s1 *= inv_c;
    s2 *= inv_c;
    Elem<F32>* out = outs + n * a.y.sn;
#pragma unroll
    for (int v = 0; v < V; ++v) {
      const int c = (at.lane + v * at.step) * E;
      if (c < C) {
        float f[E], d[E];
        widen<F32>(x[v], f);
        widen<F32>(g[v], d);
#pragma unroll
        for (int e = 0; e < E; ++e) {
          const float xh = (f[e] - mean) * rstd;
          f[e] = rstd * (fmaf(d[e], w[v][e], -s1) - xh * s2);
        }
        store_piece<F32, ALIGNED>(out + c, narrow<F32>(f), C - c);
      }
      x[v] = xn[v];
      g[v] = gn[v];
    }
    mean = mean_n;
    rstd = rstd_n;
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
  auto go = [&](auto lanes, auto pieces, auto threads) {
    constexpr int L = decltype(lanes)::value, V = decltype(pieces)::value, T = decltype(threads)::value;
    if (grad) hipLaunchKernelGGL((norm_grad_kernel<F32, ALIGNED, L, V, T>), dim3(a.B * a.parts), dim3(s.threads), 0, stream, a);
    else hipLaunchKernelGGL((norm_kernel<F32, ALIGNED, L, V, T>), dim3(a.B * a.parts), dim3(s.threads), 0, stream, a);
  };
  using std::integral_constant;
  integral_constant<int, 0> wg;
  integral_constant<int, 1> one;
  integral_constant<int, 2> two;
  integral_constant<int, kNormThreads> few;
  if (s.lanes == 16) go(integral_constant<int, 16>{}, one, few);
  else if (s.lanes == 32) go(integral_constant<int, 32>{}, one, few);
  else if (s.lanes == 64) go(integral_constant<int, 64>{}, one, few);
  else if (s.pieces == 1) go(wg, one, few);
  else if (s.threads <= 512) go(wg, two, integral_constant<int, 512>{});
  else go(wg, two, integral_constant<int, 1024>{});
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

NormShape norm_shape(int B, int N, int C, bool grad, bool per_entry) {
  NormShape s{};
  const int pieces = (C + E - 1) / E;
  if (pieces <= 64) {
    s.lanes = pieces <= 16 ? 16 : pieces <= 32 ? 32 : 64;
    s.pieces = 1;
    s.threads = kNormThreads;
  } else {
    s.lanes = 0;
    s.pieces = pieces <= 256 ? 1 : 2;
    s.threads = ((pieces + s.pieces - 1) / s.pieces + 63) / 64 * 64;
  }
  const int rows = s.lanes ? kNormThreads / s.lanes : 1;     // of a workgroup at a time
  const int64_t full = 256 * (grad ? 4 : 8) * 256 / s.threads;   // workgroups that fill the card
  int64_t parts = (full + B - 1) / B;
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
