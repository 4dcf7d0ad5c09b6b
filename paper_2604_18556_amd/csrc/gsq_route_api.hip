// Host side of the routing in gsq_routing.h: validation and launches.
#include <hip/hip_runtime.h>

#include <cmath>

#include "gsq_check.h"
#include "gsq_route.h"

using namespace gsq;

namespace {

constexpr int32_t kMostCopies = 1024;
constexpr int64_t kMostIds = (int64_t)1 << 30, kMostTokens = (int64_t)1 << 25;

bool known_dtype(int32_t dtype) { return dtype == GSQ_DT_FP32 || sixteen_bits(dtype); }
size_t size_of(int32_t dtype) { return dtype == GSQ_DT_FP32 ? 4 : 2; }

gsq_status check_routing(const gsq_routing* r) {
  if (!r) return fail(GSQ_EINVAL, "the sizes are NULL");
  if (!known_dtype(r->dtype)) return fail(GSQ_EINVAL, "unknown dtype %d", r->dtype);
  if (r->tokens < 0 || r->tokens > kMostTokens)
    return fail(GSQ_EINVAL, "tokens must be in [0, %lld], got %lld", (long long)kMostTokens, (long long)r->tokens);
  if (r->experts < 1 || r->experts > GSQ_MAX_EXPERTS)
    return fail(GSQ_EINVAL, "experts must be in [1, %d], got %d", GSQ_MAX_EXPERTS, r->experts);
  if (r->groups < 1 || r->groups > GSQ_MAX_EXPERT_GROUPS || r->experts % r->groups)
    return fail(GSQ_EINVAL, "groups must be in [1, %d] and divide %d experts, got %d", GSQ_MAX_EXPERT_GROUPS,
                r->experts, r->groups);
  if (r->top_groups < 1 || r->top_groups > r->groups)
    return fail(GSQ_EINVAL, "top_groups must be in [1, %d], got %d", r->groups, r->top_groups);
  const int32_t left = r->top_groups * (r->experts / r->groups);
  if (r->top_k < 1 || r->top_k > GSQ_MAX_TOP_K || r->top_k > left)
    return fail(GSQ_EINVAL, "top_k must be in [1, %d], got %d", left < GSQ_MAX_TOP_K ? left : GSQ_MAX_TOP_K, r->top_k);
  if (r->score != GSQ_SCORE_SOFTMAX && r->score != GSQ_SCORE_SIGMOID)
    return fail(GSQ_EINVAL, "unknown score %d", r->score);
  if (r->group_score != GSQ_GROUP_MAX && r->group_score != GSQ_GROUP_TOP2)
    return fail(GSQ_EINVAL, "unknown group_score %d", r->group_score);
  if (!std::isfinite(r->scale)) return fail(GSQ_EINVAL, "scale is not finite");
  return GSQ_OK;
}

gsq_status check_exchange(const gsq_exchange* g, const int32_t* slots) {
  if (!g) return fail(GSQ_EINVAL, "the sizes are NULL");
  if (!known_dtype(g->dtype)) return fail(GSQ_EINVAL, "unknown dtype %d", g->dtype);
  GSQ_TRY(check_rows("tokens", g->tokens));
  GSQ_TRY(check_rows("rows", g->rows));
  GSQ_TRY(check_features("cols", g->cols));
  if (g->copies < 1 || g->copies > kMostCopies)
    return fail(GSQ_EINVAL, "copies must be in [1, %d], got %d", kMostCopies, g->copies);
  return check_array("slots", slots, 4, g->tokens > 0);
}

}  // namespace

extern "C" {

gsq_status gsq_route(const gsq_routing* r, const void* logits, const float* bias, int32_t* experts,
                     float* weights, hipStream_t stream) {
  clear_error();
  GSQ_TRY(check_routing(r));
  GSQ_TRY(check_array("logits", logits, size_of(r->dtype), r->tokens > 0));
  GSQ_TRY(check_array("bias", bias, 4, false));
  GSQ_TRY(check_array("experts", experts, 4, r->tokens > 0));
  GSQ_TRY(check_array("weights", weights, 4, r->tokens > 0));
  return launched(launch_route(*r, logits, bias, experts, weights, stream), "gsq_route");
}

gsq_status gsq_route_grad(const gsq_routing* r, const void* logits, const int32_t* experts,
                          const float* dweights, void* dlogits, hipStream_t stream) {
  clear_error();
  GSQ_TRY(check_routing(r));
  GSQ_TRY(check_array("logits", logits, size_of(r->dtype), r->tokens > 0));
  GSQ_TRY(check_array("experts", experts, 4, r->tokens > 0));
  GSQ_TRY(check_array("dweights", dweights, 4, r->tokens > 0));
  GSQ_TRY(check_array("dlogits", dlogits, size_of(r->dtype), r->tokens > 0));
  return launched(launch_route_grad(*r, logits, experts, dweights, dlogits, stream), "gsq_route_grad");
}

gsq_status gsq_group_rows(const int32_t* ids, int64_t count, int32_t groups, int64_t* offsets, int32_t* slots,
                          int32_t* sources, hipStream_t stream) {
  clear_error();
  if (count < 0 || count > kMostIds)
    return fail(GSQ_EINVAL, "count must be in [0, %lld], got %lld", (long long)kMostIds, (long long)count);
  if (groups < 1 || groups > GSQ_MAX_ROW_GROUPS)
    return fail(GSQ_EINVAL, "groups must be in [1, %d], got %d", GSQ_MAX_ROW_GROUPS, groups);
  GSQ_TRY(check_array("ids", ids, 4, count > 0));
  GSQ_TRY(check_array("offsets", offsets, 8, true));
  GSQ_TRY(check_array("slots", slots, 4, count > 0));
  GSQ_TRY(check_array("sources", sources, 4, count > 0));
  return launched(launch_group_rows(ids, count, groups, offsets, slots, sources, stream), "gsq_group_rows");
}

gsq_status gsq_dispatch_rows(const gsq_exchange* g, const void* x, const int32_t* slots, void* out,
                             hipStream_t stream) {
  clear_error();
  GSQ_TRY(check_exchange(g, slots));
  GSQ_TRY(check_array("x", x, size_of(g->dtype), g->tokens > 0));
  GSQ_TRY(check_array("out", out, size_of(g->dtype), g->rows > 0));
  return launched(launch_dispatch(*g, x, slots, out, stream), "gsq_dispatch_rows");
}

gsq_status gsq_combine_rows(const gsq_exchange* g, const void* rows, const int32_t* slots, const float* weights,
                            void* out, hipStream_t stream) {
  clear_error();
  GSQ_TRY(check_exchange(g, slots));
  GSQ_TRY(check_array("rows", rows, size_of(g->dtype), g->rows > 0));
  GSQ_TRY(check_array("weights", weights, 4, false));
  GSQ_TRY(check_array("out", out, size_of(g->dtype), g->tokens > 0));
  return launched(launch_combine(*g, rows, slots, weights, out, stream), "gsq_combine_rows");
}

gsq_status gsq_combine_rows_grad(const gsq_exchange* g, const void* dout, const void* rows, const int32_t* slots,
                                 const float* weights, void* drows, float* dweights, hipStream_t stream) {
  clear_error();
  GSQ_TRY(check_exchange(g, slots));
  GSQ_TRY(check_array("dout", dout, size_of(g->dtype), g->tokens > 0));
  GSQ_TRY(check_array("rows", rows, size_of(g->dtype), g->rows > 0));
  GSQ_TRY(check_array("weights", weights, 4, g->tokens > 0));
  GSQ_TRY(check_array("drows", drows, size_of(g->dtype), g->rows > 0));
  GSQ_TRY(check_array("dweights", dweights, 4, g->tokens > 0));
  return launched(launch_combine_grad(*g, dout, rows, slots, weights, drows, dweights, stream),
                  "gsq_combine_rows_grad");
}

}  // extern "C"
