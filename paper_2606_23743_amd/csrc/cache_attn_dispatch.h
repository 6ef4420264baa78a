// Which kernel a call of the attention over a paged cache takes, for one cache format.
#pragma once

#include "cache_attn_kernel.h"
#include "cache_attn_tile.h"

namespace sva {
namespace cattn {

template <int FMT, int D>
void launch_dim(const CacheAttnArgs& a, const CacheAttnShape& s, hipStream_t stream) {
  if (s.shared) {
    if (s.tiles == 4) launch_tile<FMT, D, 1>(a, s.wgs, stream);
    else launch_tile<FMT, D, 2>(a, s.wgs, stream);
  } else {
    if (s.tiles == 1) launch_wave<FMT, D, 1>(a, s.wgs, stream);
    else if (s.tiles == 2) launch_wave<FMT, D, 2>(a, s.wgs, stream);
    else launch_wave<FMT, D, 3>(a, s.wgs, stream);
  }
}

template <int FMT>
hipError_t launch_format(const CacheAttnArgs& a, const CacheAttnShape& s, hipStream_t stream) {
  switch (a.c.D) {
    case 64: launch_dim<FMT, 64>(a, s, stream); break;
    case 112: launch_dim<FMT, 112>(a, s, stream); break;
    case 128: launch_dim<FMT, 128>(a, s, stream); break;
    default: return hipErrorInvalidValue;
  }
  return hipGetLastError();
}

}  // namespace cattn
}  // namespace sva
