// Checks of arguments that the products, the routing and the adapters share.
#pragma once
#include <hip/hip_runtime.h>

#include "gsq_host.h"
#include "gsq_products.h"

namespace gsq {
namespace {

constexpr int64_t kMostRows = (int64_t)1 << 29, kMostFeatures = (int64_t)1 << 21;
constexpr int32_t kMostGroups = 65535;

#define GSQ_TRY(call)                    \
  do {                                   \
    const gsq_status st_ = (call);       \
    if (st_ != GSQ_OK) return st_;       \
  } while (0)

bool aligned(const void* p, size_t n) { return (reinterpret_cast<uintptr_t>(p) & (n - 1)) == 0; }

bool sixteen_bits(int32_t dtype) { return dtype == GSQ_DT_BF16 || dtype == GSQ_DT_FP16; }

gsq_status check_features(const char* name, int32_t n) {
  if (n < 1 || n > kMostFeatures)
    return fail(GSQ_EINVAL, "%s must be in [1, %lld], got %d", name, (long long)kMostFeatures, n);
  return GSQ_OK;
}

gsq_status check_rows(const char* name, int64_t n) {
  if (n < 0 || n > kMostRows)
    return fail(GSQ_EINVAL, "%s must be in [0, %lld], got %lld", name, (long long)kMostRows, (long long)n);
  return GSQ_OK;
}

// An array that holds elements (`any`) must have an address, aligned to them.
gsq_status check_array(const char* name, const void* p, size_t elem, bool any) {
  if (any && !p) return fail(GSQ_EINVAL, "%s is NULL", name);
  if (!aligned(p, elem)) return fail(GSQ_EINVAL, "%s is not aligned to %zu bytes", name, elem);
  return GSQ_OK;
}

// Groups of rows with their offsets.
gsq_status check_sizes(int32_t groups, int64_t rows, const int64_t* offsets) {
  if (groups < 1 || groups > kMostGroups)
    return fail(GSQ_EINVAL, "groups must be in [1, %d], got %d", kMostGroups, groups);
  GSQ_TRY(check_rows("rows", rows));
  if (!offsets && groups > 1) return fail(GSQ_EINVAL, "offsets is NULL with %d groups", groups);
  if (!aligned(offsets, 8)) return fail(GSQ_EINVAL, "offsets is not aligned to 8 bytes");
  return GSQ_OK;
}

// A launch's outcome.  Its grid is checked before anything is enqueued.
gsq_status launched(hipError_t e, const char* what) {
  if (e == hipSuccess) return GSQ_OK;
  if (e == hipErrorInvalidConfiguration) return fail(GSQ_EINVAL, "%s: more tiles than one launch holds", what);
  return gsq::hip_fail(e, what);
}

}  // namespace
}  // namespace gsq
