// The attention over a paged e4m3 cache (cache_attn_kernel.h, cache_attn_tile.h).
#include "cache_attn_dispatch.h"

namespace sva {

hipError_t launch_cache_attention_e4m3(const CacheAttnArgs& a, const CacheAttnShape& s, hipStream_t stream) {
  return cattn::launch_format<kCacheE4m3>(a, s, stream);
}

}  // namespace sva
