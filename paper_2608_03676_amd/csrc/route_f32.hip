// Routing of logits of type float.
#include "route_kernels.h"

namespace taot {

taot_status route_f32(const RouteArgs& a, hipStream_t stream) { return route_of<float>(a, stream); }

taot_status route_backward_f32(const float* dweights, const void* logits, const int32_t* ids, int64_t T, int32_t E,
                          int32_t k, float scale, uint32_t flags, void* dlogits, hipStream_t stream) {
  return backward_of<float>(dweights, logits, ids, T, E, k, scale, flags, dlogits, stream);
}

}  // namespace taot
