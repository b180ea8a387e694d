// Routing of logits of type __bf16.
#include "route_kernels.h"

namespace taot {

taot_status route_bf16(const RouteArgs& a, hipStream_t stream) { return route_of<__bf16>(a, stream); }

taot_status route_backward_bf16(const float* dweights, const void* logits, const int32_t* ids, int64_t T, int32_t E,
                          int32_t k, float scale, uint32_t flags, void* dlogits, hipStream_t stream) {
  return backward_of<__bf16>(dweights, logits, ids, T, E, k, scale, flags, dlogits, stream);
}

}  // namespace taot
