// The attention over a paged int8 cache (cache_attn_kernel.h, cache_attn_tile.h).
#include "cache_attn_dispatch.h"

namespace sva {

hipError_t launch_cache_attention_int8(const CacheAttnArgs& a, const CacheAttnShape& s, hipStream_t stream) {
  return cattn::launch_format<kCacheInt8>(a, s, stream);
}

}  // namespace sva
