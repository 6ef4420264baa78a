// Shape and dispatch of the attention over a paged cache, and the join of divided
// segments.
#include "cache_attn_common.h"

namespace sva {
namespace cattn {
namespace {

// The partial results of one 16-row tile's channels (one of the four that a lane
// row splits into) of a divided segment, joined in the order of the workgroups.  Bound by
// latency (lengths, then the parts, then their sums in LDS): 4 to 7 us for up to 48 rows, 12 for
// 192 of 8 sequences (34 MB of parts).
constexpr int kJoinGroups = 4;

template <int D>
__global__ __launch_bounds__(64 * kJoinGroups) void cache_join_kernel(CacheAttnArgs a, int grid_n, int nt, int max_tiles, bool by_run) {
  using PT = Part<D>;
  constexpr int JT = PT::JT;
  const int RPT = 16 * nt;                         // rows of a segment
  __shared__ __attribute__((aligned(16))) float so[kJoinGroups][64][JT];
  __shared__ float sm[kJoinGroups][16], sl[kJoinGroups][16];
  const int lane = threadIdx.x & 63, g = lane >> 4, i16 = lane & 15;
  const int grp = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  int id = blockIdx.x;
  const int w = id % kWaves;
  id /= kWaves;
  const int qt = id % nt;
  id /= nt;
  const Finder fd(a, RPT, grid_n);
  const int64_t W = fd.total;
  const int n = (int)min((int64_t)grid_n, W);
  int b, h, rt;
  int64_t base;                                    // the entry's first place
  Entry en;
  if (by_run) {                                    // the segment inside which run id + 1 begins
    if (id + 1 >= n) return;
    const int64_t x = uniform(run_of(id + 1, n, W));
    en = fd.locate(x, -1, b, base);
    const int s = uniform((int)div_floor(x - base, en.span));
    h = uniform(s / en.tiles);
    rt = s - h * en.tiles;
  } else {
    rt = id % max_tiles;
    id /= max_tiles;
    h = id % a.c.heads;
    en = fd.locate(0, id / a.c.heads, b, base);
    if (rt >= en.tiles) return;
  }
  if (rt * RPT + qt * 16 >= en.cnt * a.G) return;
  const int64_t seg = (int64_t)h * en.tiles + rt;
  const int i0 = uniform(owner(base + place_of(en, seg, 0), n, W));
  const int i1 = uniform(owner(base + place_of(en, seg, en.units - 1), n, W));
  if (i0 == i1) return;                            // one workgroup had it all, and wrote it
  if (by_run && i0 != blockIdx.x / (nt * kWaves)) return;   // the first run that begins inside it joins it

  auto slot = [&](int i) { return 2 * i + (i == i0 ? 1 : 0); };   // i0's run holds the segment's first unit
  float m = -INFINITY, l = 0.0f;
  float y[JT] = {};
  constexpr int UN = 4;
  for (int k0 = i0 + grp; k0 <= i1; k0 += kJoinGroups * UN) {
    float4 p[UN][JT / 4];
    float pm[UN], pl[UN];
#pragma unroll
    for (int k = 0; k < UN; ++k) {
      const int i = min(k0 + k * kJoinGroups, i1);
      const float* part = a.ws + (int64_t)slot(i) * PT::floats(nt);
      const float* from = part + PT::at(qt, w, lane);
#pragma unroll
      for (int j = 0; j < JT / 4; ++j) p[k][j] = *reinterpret_cast<const float4*>(from + 4 * j);
      pm[k] = part[PT::ref(nt, qt * 16 + i16)];
      pl[k] = part[PT::sum(nt, qt * 16 + i16)];
    }
#pragma unroll
    for (int k = 0; k < UN; ++k) {
      if (k0 + k * kJoinGroups > i1) break;
      const float to = fmaxf(m, pm[k]);
      const float ref = to == -INFINITY ? 0.0f : to;
      const float f0 = __builtin_amdgcn_exp2f(m - ref), f1 = __builtin_amdgcn_exp2f(pm[k] - ref);
      m = to;
      l = l * f0 + pl[k] * f1;
#pragma unroll
      for (int j = 0; j < JT / 4; ++j) {
        y[4 * j] = y[4 * j] * f0 + p[k][j].x * f1;
        y[4 * j + 1] = y[4 * j + 1] * f0 + p[k][j].y * f1;
        y[4 * j + 2] = y[4 * j + 2] * f0 + p[k][j].z * f1;
        y[4 * j + 3] = y[4 * j + 3] * f0 + p[k][j].w * f1;
      }
    }
  }
#pragma unroll
  for (int j = 0; j < JT; ++j) so[grp][lane][j] = y[j];
  if (g == 0) {
    sm[grp][i16] = m;
    sl[grp][i16] = l;
  }
  __syncthreads();
  if (grp != 0) return;
  float top = sm[0][i16];
#pragma unroll
  for (int k = 1; k < kJoinGroups; ++k) top = fmaxf(top, sm[k][i16]);
  const float ref = top == -INFINITY ? 0.0f : top;
  l = 0.0f;
#pragma unroll
  for (int j = 0; j < JT; ++j) y[j] = 0.0f;
#pragma unroll
  for (int k = 0; k < kJoinGroups; ++k) {
    const float f = __builtin_amdgcn_exp2f(sm[k][i16] - ref);
    l += sl[k][i16] * f;
#pragma unroll
    for (int j = 0; j < JT; ++j) y[j] += so[k][lane][j] * f;
  }
  const int row = rt * RPT + qt * 16 + i16;
  const int t = row / a.G, head = h * a.G + (row - t * a.G);
  if (t >= en.cnt) return;
  const float inv = 1.0f / l;
#pragma unroll
  for (int j = 0; j < JT; ++j) y[j] = l == 0.0f ? 0.0f : y[j] * inv;
  const int d0 = JT * (4 * g + w);
  if (d0 < D) store_row<D>(a, b, head, t, d0, y);
  if (a.lse && w == 0 && g == 0)
    a.lse[((int64_t)b * a.H + head) * a.T + t] = l == 0.0f ? -INFINITY : (top + __log2f(l)) * kLn2;
}

template <int D>
void launch_join(const CacheAttnArgs& a, const CacheAttnShape& s, hipStream_t stream) {
  const int segments = (int)(((int64_t)a.G * a.T + 16 * s.tiles - 1) / (16 * s.tiles));
  // Only segments that several workgroups share are joined, each with at least one run that begins
  // inside it: where there are fewer runs than segments, those are looked at (1,024 sequences of up
  // to 1,000 e4m3 tokens, 8 cache heads: a call of 840 us became 205, with the sums of many
  // entries by lane)
  const int64_t all = (int64_t)a.B * a.c.heads * segments;
  const bool by_run = all > s.wgs - 1;
  const dim3 grid((unsigned)((by_run ? s.wgs - 1 : all) * s.tiles * kWaves));
  hipLaunchKernelGGL(cache_join_kernel<D>, grid, dim3(64 * kJoinGroups), 0, stream, a, s.wgs, s.tiles, segments, by_run);
}

}  // namespace
}  // namespace cattn

CacheAttnShape cache_attn_shape(const CacheAttnArgs& a) {
  using namespace cattn;
  constexpr int kCus = 256;
  CacheAttnShape s{};
  const int64_t rows = (int64_t)a.G * a.T;
  // Up to three 16-row tiles each wave holds the state of all rows and has keys of its
  // own; past that the registers do not, and the waves share keys and divide rows.  us, own keys /
  // shared ones, bf16 results: two sequences of 223,200 and 8 cache heads, 30 rows 191 / 241 (e4m3), 289 / 290
  // (bf16 cache), 48 rows 199 / 230, 317 / 289; eight of 32,768 and 6 heads, 64 rows (in two passes
  // over the keys, or one) 203 / 144 (int8), 287 / 148 (bf16), 128 rows 286 / 170, 412 / 179, 192 rows
  // 362 / 299, 510 / 313.  Float32 results: 48 rows 244 / 280, 313 / 328; 64 rows 233 / 157, 286 / 174.
  s.shared = rows > 48;
  if (s.shared) {
    const int64_t passes = (rows + 127) / 128;     // 128 rows are what a workgroup's registers hold
    s.tiles = 4 * (int)(((rows + passes - 1) / passes + 63) / 64);
  } else {
    s.tiles = (int)((rows + 15) / 16);
  }
  // as many workgroups as are resident at once
  const int resident = kCus * (s.shared ? 2 : wave_residents(a.c.D, s.tiles));
  const int cap = a.max_pages << a.c.log2_page;
  const Entry e = entry_of(cap, a.T, cap, a.T, a.G, 16 * s.tiles, true, 0);
  s.split = e.units > kWholeUnits;
  const int64_t most = (int64_t)(s.split ? e.units : 1) * e.tiles * a.c.heads * a.B;
  s.wgs = (int)(most < resident ? most : resident);
  const size_t floats = a.c.D > 64 ? Part<128>::floats(s.tiles) : Part<64>::floats(s.tiles);
  s.ws_bytes = s.split ? (size_t)2 * s.wgs * floats * 4 : 0;
  return s;
}

hipError_t launch_cache_attention(const CacheAttnArgs& args, hipStream_t stream) {
  const CacheAttnShape s = cache_attn_shape(args);
  CacheAttnArgs a = args;
  a.divide = s.split;
  hipError_t e;
  if (a.c.format == kCacheBf16) e = launch_cache_attention_bf16(a, s, stream);
  else if (a.c.format == kCacheE4m3) e = launch_cache_attention_e4m3(a, s, stream);
  else e = launch_cache_attention_int8(a, s, stream);
  if (e != hipSuccess || !s.split) return e;
  switch (a.c.D) {
    case 64: cattn::launch_join<64>(a, s, stream); break;
    case 112: cattn::launch_join<112>(a, s, stream); break;
    default: cattn::launch_join<128>(a, s, stream); break;
  }
  return hipGetLastError();
}

}  // namespace sva
