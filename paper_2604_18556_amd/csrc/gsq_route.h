// Internal declarations of the routing: experts of tokens, the order of their rows, and the rows' way there and
// back.
#pragma once
#include <hip/hip_runtime.h>
#include <stdint.h>

#include "gsq_routing.h"

namespace gsq {

hipError_t launch_route(const gsq_routing& r, const void* logits, const float* bias, int32_t* experts, float* weights,
                        hipStream_t s);
hipError_t launch_route_grad(const gsq_routing& r, const void* logits, const int32_t* experts, const float* dweights,
                             void* dlogits, hipStream_t s);
hipError_t launch_group_rows(const int32_t* ids, int64_t count, int groups, int64_t* offsets, int32_t* slots,
                             int32_t* sources, hipStream_t s);
hipError_t launch_dispatch(const gsq_exchange& g, const void* x, const int32_t* slots, void* out, hipStream_t s);
hipError_t launch_combine(const gsq_exchange& g, const void* rows, const int32_t* slots, const float* weights, void* out,
                          hipStream_t s);
hipError_t launch_combine_grad(const gsq_exchange& g, const void* dout, const void* rows, const int32_t* slots,
                               const float* weights, void* drows, float* dweights, hipStream_t s);

}  // namespace gsq
