// Internal declarations of the low-rank adapters.
#pragma once
#include <hip/hip_runtime.h>
#include <stdint.h>

#include "gsq_adapters.h"
#include "gsq_product.h"

namespace gsq {

// rows.groups are the segments; O, I, q (rank) as in gsq_adapters.h.
struct AdapterArgs {
  GroupRows rows;
  const int32_t* index;
  const float* scales;
  int32_t adapters, O, I, q;
  const void *x, *dy, *a, *b, *base;
  float* hidden;               // also dhidden
  const float *h, *dh;         // what the weights' gradients read
  void* out;
  void *da, *db;
  int32_t out_dtype, accumulate;
  int32_t vector_hidden;       // hidden may be stored four at a time
};

hipError_t launch_adapter_rows(int form, int dtype, const AdapterArgs& p, hipStream_t s);   // kForward, kInputGrad
hipError_t launch_adapter_weights(int dtype, const AdapterArgs& p, hipStream_t s);

}  // namespace gsq
