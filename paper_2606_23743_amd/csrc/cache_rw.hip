// Writing K and V rows into a paged cache (bf16, e4m3 or int8 with a scale per
// token and head) and reading them back.
//
// A cache holds [page][head][place][D] codes, so a head's tokens of a page lie
// together: the attention over it reads whole lines in order.  Both kernels are
// bound by HBM (each row read once, written once); a row is owned by 16 lanes (8
// when D = 64) of 8 channels, one 16-byte access of bf16 and one 8-byte access of
// codes.  A workgroup takes 16 (32) consecutive tokens of four heads: the four
// heads' 1 KB of a token-major input lie together, and so do the codes of
// the consecutive tokens of one head; a token's slot is looked up once for its
// four rows, all of which are loaded before the first is used.
#include <type_traits>

#include "sva_internal.h"

namespace sva {
namespace {

constexpr int kThreads = 256;
constexpr int kHeads = 4;        // heads of a workgroup

typedef __attribute__((ext_vector_type(2))) unsigned u32x2;
typedef __attribute__((ext_vector_type(4))) unsigned u32x4;
typedef __attribute__((ext_vector_type(2))) float f32x2;
typedef __attribute__((ext_vector_type(2))) __bf16 bf16x2;

// Calls past the caches (64 MB) are streamed where that pays; us, plain / non-temporal: 8-bit
// codes of bf16 rows 138 / 129 (111,600 tokens of 8 heads of 128), 60 / 56 (50,000 of 16 of 64);
// of float32 rows, and bf16 rows as they are, 188 / 192 and 149 / 152.  Reading back
// as float32, stores only: 82 / 69 (15,602 of 20 of 112), 200 / 192 (50,000 of 16); as bf16
// 132 / 136 and 118 / 114.
template <bool NT, class T>
__device__ __forceinline__ T load(const T* p) {
  if constexpr (NT) return __builtin_nontemporal_load(p);
  return *p;
}
template <bool NT, class T>
__device__ __forceinline__ void store(T* p, T v) {
  if constexpr (NT) __builtin_nontemporal_store(v, p);
  else *p = v;
}

__device__ __forceinline__ float lo16(uint32_t w) { return __uint_as_float(w << 16); }
__device__ __forceinline__ float hi16(uint32_t w) { return __uint_as_float(w & 0xFFFF0000u); }
__device__ __forceinline__ uint32_t pack_bf16(float a, float b) {
  const f32x2 f = {a, b};
  return __builtin_bit_cast(uint32_t, __builtin_convertvector(f, bf16x2));   // nearest, ties to even
}

// the largest of a row's TPR lanes, in each of them (DPP lane moves)
template <int TPR>
__device__ __forceinline__ float row_max(float x) {
  auto take = [&](auto ctrl) {
    x = fmaxf(x, __int_as_float(
                     __builtin_amdgcn_update_dpp(0, __float_as_int(x), decltype(ctrl)::value, 0xf, 0xf, true)));
  };
  if constexpr (TPR == 16) {                   // rotations of the 16 lanes by 8, 4, 2, 1
    take(std::integral_constant<int, 0x128>{});
    take(std::integral_constant<int, 0x124>{});
    take(std::integral_constant<int, 0x122>{});
    take(std::integral_constant<int, 0x121>{});
  } else {                                     // pairs, quads, then the mirrored eight lanes
    take(std::integral_constant<int, 0xB1>{});
    take(std::integral_constant<int, 0x4E>{});
    take(std::integral_constant<int, 0x141>{});
  }
  return x;
}

// smallest e in [-127, 127] with amax <= 448 * 2^e; 0 for amax = 0
// (448 = 0.875 * 2^9 and amax = f * 2^x with f in [0.5, 1))
__device__ __forceinline__ int e4m3_exp(float amax) {
  if (!(amax > 0.0f)) return 0;
  int x;
  const float f = frexpf(amax, &x);
  const int e = f <= 0.875f ? x - 9 : x - 8;
  return e < -127 ? -127 : (e > 127 ? 127 : e);
}

// Eight x / s to the nearest whole numbers, ties to even, as bytes.  x times the rounded
// reciprocal, plus 1.5 * 2^23, has the whole number in its low bits; it may be one off next to
// a half step, which the exact residual x - k s shows (its difference from s/2 is a multiple
// of ulp(s)/2: one fma holds it).  Residuals below half a step prove all eight right; else,
// rarely, each is looked at.  (Looked at every time, the instructions bound the kernel: 108 us
// for 2 x 16,380 tokens of 20 heads of 112.)
__device__ __forceinline__ u32x2 int8_codes(const float (&x)[8], float s, bool lifted) {
  constexpr float kWhole = 12582912.0f;
  const float inv = 1.0f / s, half = 0.5f * s;
  float t[8], far = 0.0f;
#pragma unroll
  for (int e = 0; e < 8; ++e) {
    t[e] = fmaf(x[e], inv, kWhole);
    far = fmaxf(far, fabsf(fmaf(-(t[e] - kWhole), s, x[e])));
  }
  if (__builtin_expect(__builtin_amdgcn_ballot_w64(far >= half || lifted) != 0, 0)) {
    asm volatile("");                          // a branch that is rarely taken, not selects
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      float k = rintf(x[e] * inv);
      const float r = fmaf(-k, s, x[e]);
      const bool odd = ((int)k & 1) != 0;
      if (fabsf(r) > half || (fabsf(r) == half && odd)) k += copysignf(1.0f, r);
      t[e] = fminf(fmaxf(k, -127.0f), 127.0f) + kWhole;
    }
  }
  u32x2 o;
#pragma unroll
  for (int w = 0; w < 2; ++w) {
    const uint32_t lo = __builtin_amdgcn_perm(__float_as_uint(t[4 * w + 1]), __float_as_uint(t[4 * w]), 0x0c0c0400u);
    const uint32_t hi = __builtin_amdgcn_perm(__float_as_uint(t[4 * w + 3]), __float_as_uint(t[4 * w + 2]), 0x04000c0cu);
    o[w] = lo | hi;
  }
  return o;
}

// eight values -> codes and the row's scale (every lane of the row has it)
template <int FMT, int TPR>
__device__ __forceinline__ u32x2 quantise8(const float (&y)[8], float& scale) {
  float m = 0.0f;
#pragma unroll
  for (int e = 0; e < 8; ++e) m = fmaxf(m, fabsf(y[e]));
  m = row_max<TPR>(m);
  u32x2 o;
  if constexpr (FMT == kCacheE4m3) {
    const int e = e4m3_exp(m);
    scale = ldexpf(1.0f, e);
    const float inv = ldexpf(1.0f, -e);        // exact products
#pragma unroll
    for (int w = 0; w < 2; ++w) {
      int c = 0;
      c = __builtin_amdgcn_cvt_pk_fp8_f32(y[4 * w] * inv, y[4 * w + 1] * inv, c, false);
      c = __builtin_amdgcn_cvt_pk_fp8_f32(y[4 * w + 2] * inv, y[4 * w + 3] * inv, c, true);
      o[w] = (uint32_t)c;
    }
  } else {
    scale = m / 127.0f;
    if (!(scale > 0.0f)) scale = 1.0f;
    // tiny rows are lifted by a power of two, so that the reciprocal is finite
    const bool lifted = scale < 0x1p-100f;
    if (__builtin_expect(__builtin_amdgcn_ballot_w64(lifted) != 0, 0)) {
      const float lift = lifted ? 0x1p100f : 1.0f;
      float z[8];
#pragma unroll
      for (int e = 0; e < 8; ++e) z[e] = y[e] * lift;
      o = int8_codes(z, scale * lift, true);
    } else {
      o = int8_codes(y, scale, false);
    }
  }
  return o;
}

// eight codes -> values times scale
template <int FMT>
__device__ __forceinline__ void widen8(u32x2 c, float scale, float (&y)[8]) {
#pragma unroll
  for (int w = 0; w < 2; ++w) {
    if constexpr (FMT == kCacheE4m3) {
      const f32x2 a = __builtin_amdgcn_cvt_pk_f32_fp8((int)c[w], false);
      const f32x2 b = __builtin_amdgcn_cvt_pk_f32_fp8((int)c[w], true);
      y[4 * w] = a[0] * scale;
      y[4 * w + 1] = a[1] * scale;
      y[4 * w + 2] = b[0] * scale;
      y[4 * w + 3] = b[1] * scale;
    } else {
#pragma unroll
      for (int e = 0; e < 4; ++e) y[4 * w + e] = (float)((int)(c[w] << (24 - 8 * e)) >> 24) * scale;
    }
  }
}

// where a workgroup's lane works: its row of tokens, its slot, its chunk
template <int D>
struct Place {
  static constexpr int TPR = D == 64 ? 8 : 16;
  static constexpr int RPP = kThreads / TPR;   // tokens of a workgroup
  static constexpr int NCH = D / 8;
  int b, n, h0, chunk;
  bool here, live;                             // the token exists; the chunk holds channels (D = 112: 14 of 16)
  int64_t row;                                 // element offset of (slot, head h0) in codes over D, or -1
  int64_t head_step;                           // rows between heads of a page

  __device__ __forceinline__ Place(const CacheRowsArgs& a) {
    const int groups = (a.c.heads + kHeads - 1) / kHeads;
    const int wg = a.first + xcd_remap(blockIdx.x, gridDim.x);
    const int tile = wg / groups;
    h0 = (wg - tile * groups) * kHeads;
    const int r = threadIdx.x / TPR;
    chunk = threadIdx.x - r * TPR;
    live = chunk < NCH;
    if (!live) chunk = 0;
    int64_t t = (int64_t)tile * RPP + r;
    const int64_t all = (int64_t)a.B * a.N;
    here = t < all;
    if (!here) t = all - 1;
    b = (int)(t / a.N);
    n = (int)(t - (int64_t)b * a.N);
    const int slot = a.slots[(int64_t)b * a.slots_b + n];
    head_step = (int64_t)1 << a.c.log2_page;
    const int page = slot >> a.c.log2_page;
    row = slot < 0 || page >= a.c.num_pages
              ? -1 : ((int64_t)page * a.c.heads + h0) * head_step + (slot & ((1 << a.c.log2_page) - 1));
  }
};

template <int D, int FMT, bool F32, bool NT>
__global__ __launch_bounds__(kThreads) void cache_write_kernel(CacheRowsArgs a) {
  using P = Place<D>;
  const P p(a);
  const bool isv = blockIdx.y != 0;
  const HeadsView x = isv ? a.v : a.k;
  const int64_t from = p.b * x.sb + p.n * x.sn + p.chunk * 8;
  u32x4 w[kHeads][F32 ? 2 : 1];
#pragma unroll
  for (int u = 0; u < kHeads; ++u) {
    const int h = min(p.h0 + u, a.c.heads - 1);
    const int64_t at = from + h * x.sh;
    if constexpr (F32) {
      w[u][0] = load<NT>(reinterpret_cast<const u32x4*>(static_cast<const float*>(x.p) + at));
      w[u][1] = load<NT>(reinterpret_cast<const u32x4*>(static_cast<const float*>(x.p) + at + 4));
    } else {
      w[u][0] = load<NT>(reinterpret_cast<const u32x4*>(static_cast<const uint16_t*>(x.p) + at));
    }
  }
  const bool put = p.here && p.row >= 0;
#pragma unroll
  for (int u = 0; u < kHeads; ++u) {
    if (p.h0 + u >= a.c.heads) break;          // uniform
    const int64_t row = p.row + u * p.head_step;
    float y[8];
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      if constexpr (F32) {
        y[e] = __uint_as_float(w[u][0][e]);
        y[4 + e] = __uint_as_float(w[u][1][e]);
      } else {
        y[2 * e] = lo16(w[u][0][e]);
        y[2 * e + 1] = hi16(w[u][0][e]);
      }
    }
    void* codes = isv ? a.c.v : a.c.k;
    if constexpr (FMT == kCacheBf16) {
      u32x4 o;
#pragma unroll
      for (int e = 0; e < 4; ++e) o[e] = F32 ? pack_bf16(y[2 * e], y[2 * e + 1]) : w[u][0][e];
      if (put && p.live) *reinterpret_cast<u32x4*>(static_cast<uint16_t*>(codes) + row * D + p.chunk * 8) = o;
    } else {
      float scale;
      const u32x2 o = quantise8<FMT, P::TPR>(y, scale);
      if (put && p.live) {
        store<NT>(reinterpret_cast<u32x2*>(static_cast<uint8_t*>(codes) + row * D + p.chunk * 8), o);
        if (p.chunk == 0) (isv ? a.c.vs : a.c.ks)[row] = scale;
      }
    }
  }
}

template <int D, int FMT, bool F32, bool NT>
__global__ __launch_bounds__(kThreads) void cache_read_kernel(CacheRowsArgs a) {
  const Place<D> p(a);
  const bool isv = blockIdx.y != 0;
  const HeadsView x = isv ? a.v : a.k;
  const void* codes = isv ? a.c.v : a.c.k;
  const float* scales = isv ? a.c.vs : a.c.ks;
  const bool got = p.row >= 0;
  const int64_t row0 = got ? p.row : 0;        // a bad slot reads page 0's first heads, and gives zeros
  // A lane's eight channels: one piece; for float32 results two runs of four, so that
  // each of its two stores is contiguous over the lanes
  constexpr int R = F32 ? 2 : 1, EB = FMT == kCacheBf16 ? 2 : 1;
  using W = std::conditional_t<FMT == kCacheBf16, u32x4, u32x2>;
  W w[kHeads];
  const int at0 = F32 ? 4 * p.chunk : 8 * p.chunk, at1 = F32 ? at0 + D / 2 : at0 + 4;
  float s[kHeads];
  const int64_t last = got ? (int64_t)(a.c.heads - 1 - p.h0) * p.head_step : 0;
#pragma unroll
  for (int u = 0; u < kHeads; ++u) {
    const int64_t row = row0 + min((int64_t)u * p.head_step, last);
    const uint8_t* from = static_cast<const uint8_t*>(codes) + row * (D * EB);
    using H = std::conditional_t<FMT == kCacheBf16, u32x2, uint32_t>;
    if constexpr (R == 1) {
      w[u] = *reinterpret_cast<const W*>(from + at0 * EB);
    } else {
      const H lo = *reinterpret_cast<const H*>(from + at0 * EB), hi = *reinterpret_cast<const H*>(from + at1 * EB);
      if constexpr (FMT == kCacheBf16) w[u] = W{lo[0], lo[1], hi[0], hi[1]};
      else w[u] = W{lo, hi};
    }
    if constexpr (FMT != kCacheBf16) s[u] = scales[row];
  }
  const int64_t to = p.b * x.sb + p.n * x.sn;
#pragma unroll
  for (int u = 0; u < kHeads; ++u) {
    if (p.h0 + u >= a.c.heads) break;          // uniform
    if (!p.here || !p.live) continue;
    const int64_t at = to + (p.h0 + u) * x.sh;
    [[maybe_unused]] float y[8];
    if constexpr (FMT == kCacheBf16) {
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        y[2 * e] = lo16(w[u][e]);
        y[2 * e + 1] = hi16(w[u][e]);
      }
    } else {
      widen8<FMT>(w[u], s[u], y);
    }
    u32x4 o[F32 ? 2 : 1];
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      if constexpr (F32) {
        o[0][e] = got ? __float_as_uint(y[e]) : 0u;
        o[1][e] = got ? __float_as_uint(y[4 + e]) : 0u;
      } else {
        uint32_t b;
        if constexpr (FMT == kCacheBf16) b = w[u][e];
        else b = pack_bf16(y[2 * e], y[2 * e + 1]);
        o[0][e] = got ? b : 0u;
      }
    }
    if constexpr (F32) {
      store<NT>(reinterpret_cast<u32x4*>(static_cast<float*>(x.p) + at + at0), o[0]);
      store<NT>(reinterpret_cast<u32x4*>(static_cast<float*>(x.p) + at + at1), o[1]);
    } else {
      store<NT>(reinterpret_cast<u32x4*>(static_cast<uint16_t*>(x.p) + at + at0), o[0]);
    }
  }
}

template <int D, int FMT, bool F32>
void launch_one(const CacheRowsArgs& args, bool write, hipStream_t stream) {
  CacheRowsArgs a = args;
  const int64_t tiles = ((int64_t)a.B * a.N + Place<D>::RPP - 1) / Place<D>::RPP;
  constexpr bool kWriteNT = FMT != kCacheBf16 && !F32, kReadNT = F32;
  const bool big = (int64_t)a.B * a.N * a.c.heads * D * (F32 ? 4 : 2) >= (64 << 20);
  launch_slices(tiles * ((a.c.heads + kHeads - 1) / kHeads), kThreads, [&](int first, unsigned n) {
    a.first = first;
    const dim3 grid(n, 2);
    if (write) {
      if (big) hipLaunchKernelGGL((cache_write_kernel<D, FMT, F32, kWriteNT>), grid, dim3(kThreads), 0, stream, a);
      else hipLaunchKernelGGL((cache_write_kernel<D, FMT, F32, false>), grid, dim3(kThreads), 0, stream, a);
    } else {
      if (big) hipLaunchKernelGGL((cache_read_kernel<D, FMT, F32, kReadNT>), grid, dim3(kThreads), 0, stream, a);
      else hipLaunchKernelGGL((cache_read_kernel<D, FMT, F32, false>), grid, dim3(kThreads), 0, stream, a);
    }
  });
}

template <int D>
hipError_t launch_rows(const CacheRowsArgs& a, bool write, hipStream_t stream) {
  switch (a.c.format * 2 + (a.f32 ? 1 : 0)) {
    case 0: launch_one<D, kCacheBf16, false>(a, write, stream); break;
    case 1: launch_one<D, kCacheBf16, true>(a, write, stream); break;
    case 2: launch_one<D, kCacheE4m3, false>(a, write, stream); break;
    case 3: launch_one<D, kCacheE4m3, true>(a, write, stream); break;
    case 4: launch_one<D, kCacheInt8, false>(a, write, stream); break;
    default: launch_one<D, kCacheInt8, true>(a, write, stream); break;
  }
  return hipGetLastError();
}

hipError_t launch_dim(const CacheRowsArgs& a, bool write, hipStream_t stream) {
  switch (a.c.D) {
    case 64: return launch_rows<64>(a, write, stream);
    case 112: return launch_rows<112>(a, write, stream);
    case 128: return launch_rows<128>(a, write, stream);
    default: return hipErrorInvalidValue;
  }
}

}  // namespace

hipError_t launch_cache_write(const CacheRowsArgs& a, hipStream_t stream) { return launch_dim(a, true, stream); }
hipError_t launch_cache_read(const CacheRowsArgs& a, hipStream_t stream) { return launch_dim(a, false, stream); }

}  // namespace sva
