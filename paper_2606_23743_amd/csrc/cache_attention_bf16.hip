// cache_attn_kernel.h over a bf16 cache.
#include "cache_attn_kernel.h"

namespace sva {
namespace cattn {

hipError_t launch_bf16(const CacheAttnArgs& a, const CacheAttnShape& s, hipStream_t stream) {
  return launch_format<kCacheBf16>(a, s, stream);
}

}  // namespace cattn
}  // namespace sva
