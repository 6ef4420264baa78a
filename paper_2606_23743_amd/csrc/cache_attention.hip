// Dispatch of the attention over a paged cache, and the join of divided segments.
#include "cache_attn_kernel.h"

namespace sva {

namespace {

constexpr int kCus = 256;

template <int D>
void launch_join(const CacheAttnArgs& a, const CacheAttnShape& s, int tiles, hipStream_t stream) {
  using namespace cattn;
  const dim3 grid((unsigned)((int64_t)a.B * a.c.heads * tiles * s.qt * kWaves));
  const dim3 block(64 * kJoinGroups);
  if (s.qt == 1) hipLaunchKernelGGL((cache_join_kernel<D, 1>), grid, block, 0, stream, a, s.wgs, tiles);
  else if (s.qt == 2) hipLaunchKernelGGL((cache_join_kernel<D, 2>), grid, block, 0, stream, a, s.wgs, tiles);
  else hipLaunchKernelGGL((cache_join_kernel<D, 4>), grid, block, 0, stream, a, s.wgs, tiles);
}

}  // namespace

CacheAttnShape cache_attn_shape(const CacheAttnArgs& a) {
  using namespace cattn;
  CacheAttnShape s{};
  const int64_t rows = (int64_t)a.G * a.T;
  s.qt = rows <= 16 ? 1 : (rows <= 32 ? 2 : 4);
  // as many workgroups as are resident at once
  const int resident = kCus * (s.qt == 1 ? 4 : 2);
  const Entry e = entry_of(a.max_pages << a.c.log2_page, a.T, a.max_pages << a.c.log2_page, a.T, a.G, 16 * s.qt, true);
  const int64_t most = entry_work(e, a.c.heads) * a.B;
  s.wgs = (int)(most < resident ? most : resident);
  s.split = e.units > 1;
  const int64_t floats = (int64_t)16 * s.qt * ((a.c.D > 64 ? 128 : 64) + 2);
  s.ws_bytes = s.split ? (size_t)(2 * s.wgs * floats * 4) : 0;
  return s;
}

hipError_t launch_cache_attention(const CacheAttnArgs& a, hipStream_t stream) {
  using namespace cattn;
  const CacheAttnShape s = cache_attn_shape(a);
  hipError_t e;
  if (a.c.format == kCacheBf16) e = launch_bf16(a, s, stream);
  else if (a.c.format == kCacheE4m3) e = launch_e4m3(a, s, stream);
  else e = launch_int8(a, s, stream);
  if (e != hipSuccess || !s.split) return e;
  const int tiles = (int)(((int64_t)a.G * a.T + 16 * s.qt - 1) / (16 * s.qt));
  switch (a.c.D) {
    case 64: launch_join<64>(a, s, tiles, stream); break;
    case 112: launch_join<112>(a, s, tiles, stream); break;
    default: launch_join<128>(a, s, tiles, stream); break;
  }
  return hipGetLastError();
}

}  // namespace sva
