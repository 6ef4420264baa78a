// cache_attn_kernel.h over a int8 cache.
#include "cache_attn_kernel.h"

namespace sva {
namespace cattn {

hipError_t launch_int8(const CacheAttnArgs& a, const CacheAttnShape& s, hipStream_t stream) {
  return launch_format<kCacheInt8>(a, s, stream);
}

}  // namespace cattn
}  // namespace sva
