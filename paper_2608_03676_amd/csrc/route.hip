// Routing by the type of the logits; the kernels are in route_kernels.h, each
// type in a file of its own.
#include "route.h"

namespace taot {

taot_status launch_route(const void* logits, const float* bias, int64_t T, int32_t E, int32_t k, int32_t groups,
                         int32_t top_groups, float scale, uint32_t flags, int32_t dtype, int32_t* ids,
                         float* weights, hipStream_t stream) {
  constexpr int64_t kMost = 1 << 22;  // tokens of a launch, of up to 256 threads each: their number has 32 bits
  auto* call = dtype == TAOT_BF16 ? route_bf16 : dtype == TAOT_F16 ? route_f16 : route_f32;
  const int64_t token_bytes = (int64_t)E * (dtype == TAOT_F32 ? 4 : 2);
  for (int64_t t = 0; t < T; t += kMost) {
    const RouteArgs a{static_cast<const char*>(logits) + t * token_bytes, bias, T - t < kMost ? T - t : kMost, E, k,
                      groups, top_groups, scale, flags, ids + t * k, weights + t * k};
    if (taot_status s = call(a, stream)) return s;
  }
  return TAOT_OK;
}

taot_status launch_route_backward(const float* dweights, const void* logits, const int32_t* ids, int64_t T,
                                  int32_t E, int32_t k, float scale, uint32_t flags, int32_t dtype, void* dlogits,
                                  hipStream_t stream) {
  auto* call = dtype == TAOT_BF16 ? route_backward_bf16 : dtype == TAOT_F16 ? route_backward_f16 : route_backward_f32;
  return call(dweights, logits, ids, T, E, k, scale, flags, dlogits, stream);
}

}  // namespace taot
