// cache_attn_kernel.h over a e4m3 cache.
#include "cache_attn_kernel.h"

namespace sva {
namespace cattn {

hipError_t launch_e4m3(const CacheAttnArgs& a, const CacheAttnShape& s, hipStream_t stream) {
  return launch_format<kCacheE4m3>(a, s, stream);
}

}  // namespace cattn
}  // namespace sva
