// Rotary positions of Q and K: pair (a, b) number i of a row at position p
// becomes m (a cos t - b sin t, a sin t + b cos t), t = p f_i (backward: -p f_i,
// the transposed map).  Half layout: pair i is (x[i], x[i + rot/2]);
// interleaved: (x[2i], x[2i + 1]).  Channels from rot on are copied, or left
// alone in place.
//
// Bound by HBM: an element is read and written once and costs two products.
// One workgroup takes a few tokens with all heads of Q and K (or several of them, where
// a head's tokens lie together), because a pair's
// angle is the same in every head: it first tabulates (m cos t, m sin t) of its
// tokens in LDS (the angle reduced modulo one turn in float64, so that positions
// of a million are as exact as small ones), then streams rows, 16 bytes an
// access, a lane's three to six items in flight together.  63,240 tokens of 40 heads of 128, half
// of each turned: 222 us, 5.8 TB/s; 2 x 7,801 float32 tokens of 40 heads of 112: 97 us, 5.8 TB/s.
#include "sva_internal.h"

namespace sva {
namespace {

constexpr int kThreads = 256;
constexpr int kTab = 2048;       // (cos, sin) entries of a workgroup
constexpr int kMaxTok = 16;      // tokens of a workgroup

typedef __attribute__((ext_vector_type(4))) unsigned u32x4;
typedef __attribute__((ext_vector_type(2))) float f32x2;
typedef __attribute__((ext_vector_type(2))) __bf16 bf16x2;

struct RotaryGrid {
  int tok, heads;                // tokens and heads of a workgroup
  bool by_head;                  // its items in the order (head, token) instead of (token, head): BY_HEAD
  int rot_items, row_items;      // items of a row that turn, and all of them
};

template <bool NT>
__device__ __forceinline__ u32x4 load16(const void* p) {
  if constexpr (NT) return __builtin_nontemporal_load(static_cast<const u32x4*>(p));
  return *static_cast<const u32x4*>(p);
}
template <bool NT>
__device__ __forceinline__ void store16(void* p, u32x4 v) {
  if constexpr (NT) __builtin_nontemporal_store(v, static_cast<u32x4*>(p));
  else *static_cast<u32x4*>(p) = v;
}

template <bool F32> struct Elem;
template <> struct Elem<false> {
  typedef uint16_t T;
  static __device__ __forceinline__ float get(T x) { return __uint_as_float((uint32_t)x << 16); }
  static __device__ __forceinline__ T put(float x) { return __builtin_bit_cast(uint16_t, (__bf16)x); }
  // 16 bytes as 8 floats and back
  static constexpr int E = 8;
  static __device__ __forceinline__ void wide(const u32x4& w, float (&y)[E]) {
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      y[2 * i] = __uint_as_float(w[i] << 16);
      y[2 * i + 1] = __uint_as_float(w[i] & 0xFFFF0000u);
    }
  }
  static __device__ __forceinline__ u32x4 narrow(const float (&y)[E]) {
    u32x4 w;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const f32x2 f = {y[2 * i], y[2 * i + 1]};
      w[i] = __builtin_bit_cast(uint32_t, __builtin_convertvector(f, bf16x2));   // nearest, ties to even
    }
    return w;
  }
};
template <> struct Elem<true> {
  typedef float T;
  static __device__ __forceinline__ float get(T x) { return x; }
  static __device__ __forceinline__ T put(float x) { return x; }
  static constexpr int E = 4;
  static __device__ __forceinline__ void wide(const u32x4& w, float (&y)[E]) {
#pragma unroll
    for (int i = 0; i < 4; ++i) y[i] = __uint_as_float(w[i]);
  }
  static __device__ __forceinline__ u32x4 narrow(const float (&y)[E]) {
    u32x4 w;
#pragma unroll
    for (int i = 0; i < 4; ++i) w[i] = __float_as_uint(y[i]);
    return w;
  }
};

template <bool F32, bool HALF, bool VEC, int kUnroll, bool NT, bool BY_HEAD>
__global__ __launch_bounds__(kThreads) void rotary_kernel(RotaryArgs a, RotaryGrid gr) {
  using El = Elem<F32>;
  using T = typename El::T;
  constexpr int E = VEC ? El::E : 1;
  __shared__ float2 tab[kTab];
  __shared__ int64_t base[kMaxTok][4];         // offsets of a token in q_in, q_out, k_in, k_out

  const int np = a.rot / 2;
  const int t0 = blockIdx.x * gr.tok;
  const int nt = min(gr.tok, a.B * a.N - t0);
  if (threadIdx.x < nt) {
    const int b = (t0 + threadIdx.x) / a.N;
    const int64_t n = t0 + threadIdx.x - b * a.N;
    base[threadIdx.x][0] = b * a.qi.sb + n * a.qi.sn;
    base[threadIdx.x][1] = b * a.qo.sb + n * a.qo.sn;
    base[threadIdx.x][2] = b * a.ki.sb + n * a.ki.sn;
    base[threadIdx.x][3] = b * a.ko.sb + n * a.ko.sn;
  }
  for (int e = threadIdx.x; e < nt * np; e += kThreads) {
    const int tk = e / np, p = e - tk * np;
    const int b = (t0 + tk) / a.N, n = t0 + tk - b * a.N;
    double turn = (double)a.pos[b * a.pos_b + n] * (a.freq[p] * 0.15915494309189533576888);   // 1 / 2pi
    turn -= rint(turn);
    float sn, cs;
    sincospif(2.0f * (float)turn, &sn, &cs);
    tab[e] = make_float2(cs * a.magnitude, (a.backward ? -sn : sn) * a.magnitude);
  }
  __syncthreads();

  const int h0 = BY_HEAD ? blockIdx.y * gr.heads : 0;
  const int all = a.qi.heads + a.ki.heads, heads = BY_HEAD ? min(gr.heads, all - h0) : all;
  const int items = nt * heads * gr.row_items;
  const unsigned inner = BY_HEAD ? nt : heads;
  for (int i0 = 0; i0 < items; i0 += kThreads * kUnroll) {
    const T* src[kUnroll];
    T* dst[kUnroll];
    const float2* cs[kUnroll];
    int c[kUnroll];
#pragma unroll
    for (int u = 0; u < kUnroll; ++u) {
      // lanes past the end load the last item and store nothing
      const unsigned idx = min(i0 + u * kThreads + (int)threadIdx.x, items - 1);
      const unsigned row = idx / (unsigned)gr.row_items;
      c[u] = idx - row * gr.row_items;
      const unsigned far = row / inner, near = row - far * inner;
      const unsigned tk = BY_HEAD ? near : far;
      const int h = h0 + (int)(BY_HEAD ? far : near);
      const bool isq = h < a.qi.heads;
      const int hh = isq ? h : h - a.qi.heads;
      src[u] = (const T*)(isq ? a.qi.p : a.ki.p) + base[tk][isq ? 0 : 2] + hh * (isq ? a.qi.sh : a.ki.sh);
      dst[u] = (T*)(isq ? a.qo.p : a.ko.p) + base[tk][isq ? 1 : 3] + hh * (isq ? a.qo.sh : a.ko.sh);
      cs[u] = tab + tk * np;
    }
    auto live = [&](int u) { return i0 + u * kThreads + (int)threadIdx.x < items; };
    if constexpr (VEC) {
      u32x4 w[kUnroll][2];
      int at[kUnroll][2];                      // first channels of an item's one or two pieces
#pragma unroll
      for (int u = 0; u < kUnroll; ++u) {
        const bool turns = c[u] < gr.rot_items;
        at[u][0] = turns ? c[u] * E : a.rot + (c[u] - gr.rot_items) * E;
        at[u][1] = HALF && turns ? at[u][0] + np : at[u][0];
        w[u][0] = load16<NT>(src[u] + at[u][0]);
        if constexpr (HALF) w[u][1] = load16<NT>(src[u] + at[u][1]);
      }
#pragma unroll
      for (int u = 0; u < kUnroll; ++u) {
        if (!live(u)) continue;
        if (c[u] < gr.rot_items) {
          float y[E], z[E];
          El::wide(w[u][0], y);
          if constexpr (HALF) {
            El::wide(w[u][1], z);
#pragma unroll
            for (int e = 0; e < E; ++e) {
              const float2 t = cs[u][c[u] * E + e];
              const float p = y[e], q = z[e];
              y[e] = p * t.x - q * t.y;
              z[e] = p * t.y + q * t.x;
            }
            store16<NT>(dst[u] + at[u][1], El::narrow(z));
          } else {
#pragma unroll
            for (int e = 0; e < E / 2; ++e) {
              const float2 t = cs[u][c[u] * (E / 2) + e];
              const float p = y[2 * e], q = y[2 * e + 1];
              y[2 * e] = p * t.x - q * t.y;
              y[2 * e + 1] = p * t.y + q * t.x;
            }
          }
          w[u][0] = El::narrow(y);
        } else if (src[u] == dst[u]) {
          continue;                            // in place: nothing to copy
        }
        store16<NT>(dst[u] + at[u][0], w[u][0]);
      }
    } else {
#pragma unroll
      for (int u = 0; u < kUnroll; ++u) {
        if (!live(u)) continue;
        if (c[u] < gr.rot_items) {             // one pair
          const int i = HALF ? c[u] : 2 * c[u], j = HALF ? c[u] + np : 2 * c[u] + 1;
          const float2 t = cs[u][c[u]];
          const float p = El::get(src[u][i]), q = El::get(src[u][j]);
          dst[u][i] = El::put(p * t.x - q * t.y);
          dst[u][j] = El::put(p * t.y + q * t.x);
        } else {
          const int i = a.rot + c[u] - gr.rot_items;
          dst[u][i] = src[u][i];
        }
      }
    }
  }
}

template <bool F32, bool HALF, bool VEC, int U>
void launch_unroll(const RotaryArgs& a, const RotaryGrid& gr, bool nt, hipStream_t stream) {
  const int64_t tokens = (int64_t)a.B * a.N;
  const int heads = a.qi.heads + a.ki.heads;
  const dim3 grid((unsigned)((tokens + gr.tok - 1) / gr.tok), (heads + gr.heads - 1) / gr.heads);
  auto go = [&](auto kernel) { hipLaunchKernelGGL(kernel, grid, dim3(kThreads), 0, stream, a, gr); };
  if (gr.by_head && nt) go(rotary_kernel<F32, HALF, VEC, U, VEC, true>);
  else if (gr.by_head) go(rotary_kernel<F32, HALF, VEC, U, false, true>);
  else if (nt) go(rotary_kernel<F32, HALF, VEC, U, VEC, false>);
  else go(rotary_kernel<F32, HALF, VEC, U, false, false>);
}

template <bool F32, bool HALF, bool VEC>
void launch_as(const RotaryArgs& a, hipStream_t stream) {
  constexpr int E = VEC ? Elem<F32>::E : 1, kItem = F32 ? 4 : 2;
  const int heads = a.qi.heads + a.ki.heads;
  RotaryGrid gr{1, heads, false, 0, 0};
  gr.rot_items = !VEC || HALF ? a.rot / 2 / E : a.rot / E;
  gr.row_items = gr.rot_items + (a.copy ? (a.D - a.rot) / E : 0);
  // Where a head's tokens lie together (not a token's heads), a workgroup takes 4 KB of each of
  // as many heads as make four items a lane; us against all heads of fewer tokens, 2 x 7,801
  // tokens of 40 heads of 112: float32 115 / 97, bf16 interleaved 85 / 57, halves 61 / 52;
  // 30,000 tokens of 40 of 128 119 / 109, of 64 61 / 57
  if (a.N > 1 && a.qi.sn < a.qi.sh && heads <= 65535) {   // (groups are blockIdx.y)
    int64_t t = 4096 / (a.D * kItem);
    t = t < kMaxTok ? (t > 1 ? t : 1) : kMaxTok;
    int64_t most = 4 * kThreads / (t * gr.row_items);
    if (most < 1) most = 1;
    const int64_t groups = (heads + most - 1) / most;
    gr.heads = (int)((heads + groups - 1) / groups);
    gr.by_head = true;
  }
  const int64_t per_token = (int64_t)gr.heads * gr.row_items;
  // Tokens of a workgroup, within the table, and items of a lane: one round of the lanes, or
  // as few as the heads of one token need, with the fewest lanes idle.  More rounds were
  // slower: 63,240 tokens of 40 heads of 128, half turned, 220 us in one, 262 in four.
  int unroll = 4;
  double best = 0.0;
  for (int u = 3; u <= 6; ++u) {
    int64_t t = (int64_t)u * kThreads / per_token;
    t = t < kMaxTok ? t : kMaxTok;
    t = t < kTab / (a.rot / 2) ? t : kTab / (a.rot / 2);
    t = t > 1 ? t : 1;
    const int64_t round = (int64_t)u * kThreads, rounds = (t * per_token + round - 1) / round;
    const double busy = (double)(t * per_token) / (double)(rounds * round);
    if (busy > best + 0.01) {
      best = busy;
      unroll = u;
      gr.tok = (int)t;
    }
  }
  // Tensors past the caches are streamed where an access covers whole lines; us, plain /
  // non-temporal, 30,000 tokens of 48 heads: interleaved bf16 of 128 130 / 122, float32 of
  // 112 223 / 210, halves bf16 of 128 136 / 123; halves of 64 (runs of 64 bytes) 71 / 79, of 112
  // 117 / 178
  const bool lines = !HALF || a.rot / 2 * kItem % 128 == 0;
  const int64_t bytes = (int64_t)a.B * a.N * (a.qi.heads + a.ki.heads) * a.D * kItem;
  const bool nt = lines && bytes >= (64 << 20);
  if constexpr (!VEC) launch_unroll<F32, HALF, VEC, 4>(a, gr, false, stream);
  else if (unroll == 3) launch_unroll<F32, HALF, VEC, 3>(a, gr, nt, stream);
  else if (unroll == 4) launch_unroll<F32, HALF, VEC, 4>(a, gr, nt, stream);
  else if (unroll == 5) launch_unroll<F32, HALF, VEC, 5>(a, gr, nt, stream);
  else launch_unroll<F32, HALF, VEC, 6>(a, gr, nt, stream);
}

template <bool F32, bool HALF>
void launch_layout(const RotaryArgs& a, hipStream_t stream) {
  if (a.vec) launch_as<F32, HALF, true>(a, stream);
  else launch_as<F32, HALF, false>(a, stream);
}

}  // namespace

hipError_t launch_rotary(const RotaryArgs& a, hipStream_t stream) {
  if (a.f32) {
    if (a.half) launch_layout<true, true>(a, stream);
    else launch_layout<true, false>(a, stream);
  } else {
    if (a.half) launch_layout<false, true>(a, stream);
    else launch_layout<false, false>(a, stream);
  }
  return hipGetLastError();
}

}  // namespace sva
