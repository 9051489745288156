// The kernels of a2d_cached_fwd.hpp and a2d_cached_wide.hpp over a cache in bf16.
#include "a2d_cached_wide.hpp"

namespace a2d {
hipError_t launch_cached_bf16(Phase ph, int hdim, const CachedArgs& a, hipStream_t s) {
  return a.tiles > 2 ? cached::go_wide_head<A2D_CACHE_BF16>(ph, hdim, a, s) : cached::go_format<A2D_CACHE_BF16>(ph, hdim, a, s);
}
}  // namespace a2d
