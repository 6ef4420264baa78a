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
#include <type_traits>

#include "sva_internal.h"

namespace sva {
namespace {

constexpr int kThreads = 256;
constexpr int kTab = 2048;       // (cos, sin) entries of a workgroup
constexpr int kMaxTok = 16;      // tokens of a workgroup

typedef __attribute__((ext_vector_type(2))) unsigned u32x2;
typedef __attribute__((ext_vector_type(4))) unsigned u32x4;
typedef u32x4 __attribute__((aligned(4))) u32x4a;   // at any dword
typedef __attribute__((ext_vector_type(2))) float f32x2;
typedef __attribute__((ext_vector_type(2))) __bf16 bf16x2;

struct RotaryGrid {
  int tok, heads;                // tokens and heads of a workgroup
  bool by_head;                  // its items in the order (head, token) instead of (token, head): BY_HEAD
  int rot_items, row_items;      // items of a row that turn, and all of them
  int first;                     // a launch's first workgroup
};

// VB bytes at p as dwords: 16, or the largest of 8, 4 and 2 that sizes and strides are multiples of.
// RAGGED: 16 bytes at any dword, where regions are multiples of four bytes and hold 16: a region's last
// piece begins so much earlier that it ends with the region, and stores what is its own.  us, by
// elements / by 8 or 4 bytes / RAGGED, bf16: 30,703 tokens of 8 heads of 112, 56 turned in halves, 80 / 25 /
// 26; 64 x 106 of 44, the same, 78 / 42 / 33; 8 x 8,403 of 18, 54 turned in pairs, 341 / 274 / 107
template <int VB, bool NT, bool RAGGED>
__device__ __forceinline__ void load_piece(const void* p, uint32_t (&w)[(VB + 3) / 4]) {
  using W = std::conditional_t<VB == 16, u32x4, std::conditional_t<VB == 8, u32x2, std::conditional_t<VB == 4, uint32_t, uint16_t>>>;
  W x;
  if constexpr (RAGGED) x = *static_cast<const u32x4a*>(p);
  else if constexpr (NT) x = __builtin_nontemporal_load(static_cast<const W*>(p));
  else x = *static_cast<const W*>(p);
  if constexpr (VB <= 4) {
    w[0] = x;
  } else {
#pragma unroll
    for (int i = 0; i < VB / 4; ++i) w[i] = x[i];
  }
}
template <int VB, bool NT, bool RAGGED>
__device__ __forceinline__ void store_piece(void* p, const uint32_t (&w)[(VB + 3) / 4]) {
  using W = std::conditional_t<VB == 16, u32x4, std::conditional_t<VB == 8, u32x2, std::conditional_t<VB == 4, uint32_t, uint16_t>>>;
  W x;
  if constexpr (VB <= 4) {
    x = (W)w[0];
  } else {
#pragma unroll
    for (int i = 0; i < VB / 4; ++i) x[i] = w[i];
  }
  if constexpr (RAGGED) *static_cast<u32x4a*>(p) = x;
  else if constexpr (NT) __builtin_nontemporal_store(x, static_cast<W*>(p));
  else *static_cast<W*>(p) = x;
}

// a piece's E elements as floats, and back (bf16: to nearest, ties to even)
template <bool F32, int E, int N>
__device__ __forceinline__ void wide(const uint32_t (&w)[N], float (&y)[E]) {
#pragma unroll
  for (int e = 0; e < E; ++e) {
    if constexpr (F32) y[e] = __uint_as_float(w[e]);
    else y[e] = __uint_as_float(e & 1 ? w[e / 2] & 0xFFFF0000u : w[e / 2] << 16);
  }
}
template <bool F32, int E, int N>
__device__ __forceinline__ void narrow(const float (&y)[E], uint32_t (&w)[N]) {
#pragma unroll
  for (int i = 0; i < N; ++i) {
    if constexpr (F32) {
      w[i] = __float_as_uint(y[i]);
    } else {
      const f32x2 f = {y[2 * i], E > 1 ? y[E > 1 ? 2 * i + 1 : 0] : 0.0f};
      w[i] = __builtin_bit_cast(uint32_t, __builtin_convertvector(f, bf16x2));
    }
  }
}

template <bool F32, bool HALF, int VB, bool RAGGED, int kUnroll, bool NT, bool BY_HEAD>
__global__ __launch_bounds__(kThreads) void rotary_kernel(RotaryArgs a, RotaryGrid gr) {
  using T = std::conditional_t<F32, float, uint16_t>;
  constexpr int E = VB / (int)sizeof(T);       // elements of a piece
  constexpr bool TWO = HALF || E == 1;         // a pair lies in two pieces
  constexpr int NW = (VB + 3) / 4;
  __shared__ float2 tab[kTab];
  __shared__ int64_t base[kMaxTok][4];         // offsets of a token in q_in, q_out, k_in, k_out

  const int np = a.rot / 2;
  const int t0 = (gr.first + blockIdx.x) * gr.tok;
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
    double at;
    if (!a.axis) {
      at = (double)a.pos[b * a.pos_b + n];
    } else {
      // a pair of no axis stays where it is
      const unsigned axis = a.axis[p];
      const int64_t i = b * a.pos_b + n * a.pos_n + axis * a.pos_a;
      at = axis >= (unsigned)a.axes ? 0.0 : a.pos_f32 ? (double)reinterpret_cast<const float*>(a.pos)[i] : (double)a.pos[i];
    }
    double turn = at * (a.freq[p] * 0.15915494309189533576888);   // 1 / 2pi
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
    [[maybe_unused]] int skip[kUnroll];        // RAGGED: a piece's first elements that another item has
    auto put = [&](T* to, const uint32_t (&x)[NW], int u) {
      if constexpr (RAGGED) {
        if (skip[u] > 0) {
#pragma unroll
          for (int i = 0; i < NW; ++i)
            if (i * (E / NW) >= skip[u]) store_piece<4, false, false>(to + i * (E / NW), {x[i]});
          return;
        }
      }
      store_piece<VB, NT, RAGGED>(to, x);
    };
    uint32_t w[kUnroll][2][NW];
    int at[kUnroll][2];                        // first channels of an item's one or two pieces
#pragma unroll
    for (int u = 0; u < kUnroll; ++u) {
      const bool turns = c[u] < gr.rot_items;
      at[u][0] = turns ? c[u] * (TWO && !HALF ? 2 : E) : a.rot + (c[u] - gr.rot_items) * E;
      at[u][1] = TWO && turns ? at[u][0] + (HALF ? np : 1) : at[u][0];
      if constexpr (RAGGED) {
        // the region's last piece begins so much earlier that it ends with the region
        const int end = turns ? (HALF ? np : a.rot) : a.D;
        skip[u] = max(at[u][0] + E - end, 0);
        at[u][0] -= skip[u];
        at[u][1] -= skip[u];
      }
      load_piece<VB, NT, RAGGED>(src[u] + at[u][0], w[u][0]);
      if constexpr (TWO) load_piece<VB, NT, RAGGED>(src[u] + at[u][1], w[u][1]);
    }
#pragma unroll
    for (int u = 0; u < kUnroll; ++u) {
      if (!live(u)) continue;
      if (c[u] < gr.rot_items) {
        float y[E];
        wide<F32, E>(w[u][0], y);
        if constexpr (TWO) {
          float z[E];
          wide<F32, E>(w[u][1], z);
#pragma unroll
          for (int e = 0; e < E; ++e) {
            const float2 t = cs[u][(RAGGED ? at[u][0] : c[u] * E) + e];
            const float p = y[e], q = z[e];
            y[e] = p * t.x - q * t.y;
            z[e] = p * t.y + q * t.x;
          }
          narrow<F32, E>(z, w[u][1]);
          put(dst[u] + at[u][1], w[u][1], u);
        } else {
#pragma unroll
          for (int e = 0; e < E / 2; ++e) {
            const float2 t = cs[u][(RAGGED ? at[u][0] / 2 : c[u] * (E / 2)) + e];
            const float p = y[2 * e], q = y[2 * e + 1];
            y[2 * e] = p * t.x - q * t.y;
            y[2 * e + 1] = p * t.y + q * t.x;
          }
        }
        narrow<F32, E>(y, w[u][0]);
      } else if (src[u] == dst[u]) {
        continue;                              // in place: nothing to copy
      }
      put(dst[u] + at[u][0], w[u][0], u);
    }
  }
}

template <bool F32, bool HALF, int VB, bool RAGGED, int U>
void launch_unroll(const RotaryArgs& a, const RotaryGrid& grid, bool nt, hipStream_t stream) {
  RotaryGrid gr = grid;
  const int64_t tokens = (int64_t)a.B * a.N;
  const int heads = a.qi.heads + a.ki.heads;
  auto go = [&](auto kernel) {
    launch_slices((tokens + gr.tok - 1) / gr.tok, kThreads, [&](int first, unsigned n) {
      gr.first = first;
      hipLaunchKernelGGL(kernel, dim3(n, (heads + gr.heads - 1) / gr.heads), dim3(kThreads), 0, stream, a, gr);
    });
  };
  constexpr bool NT = VB == 16 && !RAGGED;
  if (gr.by_head && nt) go(rotary_kernel<F32, HALF, VB, RAGGED, U, NT, true>);
  else if (gr.by_head) go(rotary_kernel<F32, HALF, VB, RAGGED, U, false, true>);
  else if (nt) go(rotary_kernel<F32, HALF, VB, RAGGED, U, NT, false>);
  else go(rotary_kernel<F32, HALF, VB, RAGGED, U, false, false>);
}

template <bool F32, bool HALF, int VB, bool RAGGED = false>
void launch_as(const RotaryArgs& a, hipStream_t stream) {
  constexpr int kItem = F32 ? 4 : 2, E = VB / kItem;
  constexpr bool TWO = HALF || E == 1;
  const int heads = a.qi.heads + a.ki.heads;
  RotaryGrid gr{1, heads, false, 0, 0, 0};
  gr.rot_items = ((TWO ? a.rot / 2 : a.rot) + E - 1) / E;
  gr.row_items = gr.rot_items + (a.copy ? (a.D - a.rot + E - 1) / E : 0);
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
  constexpr int kOnly = RAGGED ? 4 : 6;
  for (int u = VB < 16 || RAGGED ? kOnly : 3; u <= (RAGGED ? kOnly : 6); ++u) {
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
  if constexpr (VB < 16 || RAGGED) launch_unroll<F32, HALF, VB, RAGGED, kOnly>(a, gr, false, stream);
  else if (unroll == 3) launch_unroll<F32, HALF, VB, false, 3>(a, gr, nt, stream);
  else if (unroll == 4) launch_unroll<F32, HALF, VB, false, 4>(a, gr, nt, stream);
  else if (unroll == 5) launch_unroll<F32, HALF, VB, false, 5>(a, gr, nt, stream);
  else launch_unroll<F32, HALF, VB, false, 6>(a, gr, nt, stream);
}

template <bool F32, bool HALF>
void launch_layout(const RotaryArgs& a, hipStream_t stream) {
  if (a.piece == 16) launch_as<F32, HALF, 16>(a, stream);
  else if (a.ragged) launch_as<F32, HALF, 16, true>(a, stream);
  else if (a.piece == 8) launch_as<F32, HALF, 8>(a, stream);
  else if (F32 || a.piece == 4) launch_as<F32, HALF, 4>(a, stream);
  else if constexpr (!F32) launch_as<F32, HALF, 2>(a, stream);
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
