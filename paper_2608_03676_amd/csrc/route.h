// The routing calls of one type of logits each.
#pragma once

#include "common.h"

namespace taot {

struct RouteArgs {
  const void* logits;
  const float* bias;
  int64_t T;
  int32_t E, k, groups, top_groups;
  float scale;
  uint32_t flags;
  int32_t* ids;
  float* weights;
};

taot_status route_bf16(const RouteArgs& a, hipStream_t stream);
taot_status route_f16(const RouteArgs& a, hipStream_t stream);
taot_status route_f32(const RouteArgs& a, hipStream_t stream);

taot_status route_backward_bf16(const float* dweights, const void* logits, const int32_t* ids, int64_t T, int32_t E,
                                int32_t k, float scale, uint32_t flags, void* dlogits, hipStream_t stream);
taot_status route_backward_f16(const float* dweights, const void* logits, const int32_t* ids, int64_t T, int32_t E,
                               int32_t k, float scale, uint32_t flags, void* dlogits, hipStream_t stream);
taot_status route_backward_f32(const float* dweights, const void* logits, const int32_t* ids, int64_t T, int32_t E,
                               int32_t k, float scale, uint32_t flags, void* dlogits, hipStream_t stream);

}  // namespace taot
