// Host side of the adapters in gsq_adapters.h: validation and launches.
#include <hip/hip_runtime.h>

#include "gsq_adapter.h"
#include "gsq_check.h"

using namespace gsq;

namespace {

// Sizes, and the arrays that every call has.
gsq_status check_adapters(const gsq_adapters* g, const int64_t* offsets, const int32_t* index, const float* scales) {
  if (!g) return fail(GSQ_EINVAL, "the sizes are NULL");
  if (!sixteen_bits(g->dtype)) return fail(GSQ_EINVAL, "dtype must be BF16 or FP16, got %d", g->dtype);
  GSQ_TRY(check_features("in_features", g->in_features));
  GSQ_TRY(check_features("out_features", g->out_features));
  if (g->rank < 1 || g->rank > GSQ_MAX_RANK)
    return fail(GSQ_EINVAL, "rank must be in [1, %d], got %d", GSQ_MAX_RANK, g->rank);
  if (g->adapters < 1 || g->adapters > kMostGroups)
    return fail(GSQ_EINVAL, "adapters must be in [1, %d], got %d", kMostGroups, g->adapters);
  if (g->segments < 1 || g->segments > kMostGroups)
    return fail(GSQ_EINVAL, "segments must be in [1, %d], got %d", kMostGroups, g->segments);
  GSQ_TRY(check_sizes(g->segments, g->rows, offsets));
  if (!index && g->adapters != g->segments)
    return fail(GSQ_EINVAL, "index is NULL with %d adapters for %d segments", g->adapters, g->segments);
  GSQ_TRY(check_array("index", index, 4, false));
  return check_array("scales", scales, 4, false);
}

AdapterArgs adapter_args(const gsq_adapters* g, const int64_t* offsets, const int32_t* index, const float* scales) {
  AdapterArgs p{};
  p.rows = {offsets, g->rows, g->segments};
  p.index = index;
  p.scales = scales;
  p.adapters = g->adapters;
  p.O = g->out_features;
  p.I = g->in_features;
  p.q = g->rank;
  return p;
}

}  // namespace

extern "C" {

gsq_status gsq_adapter_forward(const gsq_adapters* g, const void* x, const void* a, const void* b,
                               const int64_t* offsets, const int32_t* index, const float* scales,
                               const void* base, float* hidden, void* y, hipStream_t stream) {
  clear_error();
  GSQ_TRY(check_adapters(g, offsets, index, scales));
  GSQ_TRY(check_array("x", x, 2, g->rows > 0));
  GSQ_TRY(check_array("a", a, 2, true));
  GSQ_TRY(check_array("b", b, 2, true));
  GSQ_TRY(check_array("base", base, 2, false));
  GSQ_TRY(check_array("hidden", hidden, 4, g->rows > 0));
  GSQ_TRY(check_array("y", y, 2, g->rows > 0));
  AdapterArgs p = adapter_args(g, offsets, index, scales);
  p.x = x;
  p.a = a;
  p.b = b;
  p.base = base;
  p.hidden = hidden;
  p.out = y;
  return launched(launch_adapter_rows(kForward, g->dtype, p, stream), "gsq_adapter_forward");
}

gsq_status gsq_adapter_input_grad(const gsq_adapters* g, const void* dy, const void* a, const void* b,
                                  const int64_t* offsets, const int32_t* index, const float* scales,
                                  const void* base, float* dhidden, void* dx, hipStream_t stream) {
  clear_error();
  GSQ_TRY(check_adapters(g, offsets, index, scales));
  GSQ_TRY(check_array("dy", dy, 2, g->rows > 0));
  GSQ_TRY(check_array("a", a, 2, true));
  GSQ_TRY(check_array("b", b, 2, true));
  GSQ_TRY(check_array("base", base, 2, false));
  GSQ_TRY(check_array("dhidden", dhidden, 4, g->rows > 0));
  GSQ_TRY(check_array("dx", dx, 2, g->rows > 0));
  AdapterArgs p = adapter_args(g, offsets, index, scales);
  p.dy = dy;
  p.a = a;
  p.b = b;
  p.base = base;
  p.hidden = dhidden;
  p.out = dx;
  return launched(launch_adapter_rows(kInputGrad, g->dtype, p, stream), "gsq_adapter_input_grad");
}

gsq_status gsq_adapter_weight_grad(const gsq_adapters* g, const void* dy, const void* x, const float* hidden,
                                   const float* dhidden, const int64_t* offsets, const int32_t* index,
                                   const float* scales, void* da, void* db, int32_t dw_dtype,
                                   int32_t accumulate, hipStream_t stream) {
  clear_error();
  GSQ_TRY(check_adapters(g, offsets, index, scales));
  if (dw_dtype != g->dtype && dw_dtype != GSQ_DT_FP32)
    return fail(GSQ_EINVAL, "dw_dtype must be the type of x or FP32, got %d", dw_dtype);
  if (accumulate && dw_dtype != GSQ_DT_FP32) return fail(GSQ_EINVAL, "gradients accumulate in FP32 only");
  GSQ_TRY(check_array("dy", dy, 2, g->rows > 0));
  GSQ_TRY(check_array("x", x, 2, g->rows > 0));
  GSQ_TRY(check_array("hidden", hidden, 4, g->rows > 0));
  GSQ_TRY(check_array("dhidden", dhidden, 4, g->rows > 0));
  const size_t size = dw_dtype == GSQ_DT_FP32 ? 4 : 2;
  GSQ_TRY(check_array("da", da, size, true));
  GSQ_TRY(check_array("db", db, size, true));
  AdapterArgs p = adapter_args(g, offsets, index, scales);
  p.dy = dy;
  p.x = x;
  p.h = hidden;
  p.dh = dhidden;
  p.da = da;
  p.db = db;
  p.out_dtype = dw_dtype;
  p.accumulate = accumulate ? 1 : 0;
  return launched(launch_adapter_weights(g->dtype, p, stream), "gsq_adapter_weight_grad");
}

}  // extern "C"
