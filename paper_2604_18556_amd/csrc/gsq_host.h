// Host helpers that the files of the C ABI share: errors, configurations, device memory.
#pragma once
#include <hip/hip_runtime.h>

#include "gsq.h"
#include "gsq_pool.h"

namespace gsq {

void clear_error();   // of this thread
gsq_status fail(gsq_status st, const char* fmt, ...);
gsq_status hip_fail(hipError_t e, const char* what);
gsq_status validate_config(const gsq_config* c);
int code_bits(int n_levels);   // of a packed code

extern DevicePool g_pool;

#define GSQ_HIP(call)                                       \
  do {                                                      \
    hipError_t e_ = (call);                                 \
    if (e_ != hipSuccess) return gsq::hip_fail(e_, #call);  \
  } while (0)

}  // namespace gsq
