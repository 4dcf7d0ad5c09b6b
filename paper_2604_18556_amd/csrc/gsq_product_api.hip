// Host side of the products in gsq_products.h: validation, the packed layer's handle and launches.
#include <hip/hip_runtime.h>

#include <new>

#include "gsq_check.h"
#include "gsq_plan.h"
#include "gsq_product.h"

using namespace gsq;

struct gsq_linear {
  gsq::PackedLayer L;
  int32_t groups;
  int device;
  struct { void* p; size_t bytes; } bufs[3];
  int n_bufs;
};

namespace {

constexpr int32_t kMostExactI8 = 131071;   // 128^2 131071 < 2^31

gsq_status check_grouped(const gsq_grouped* g, const int64_t* offsets, bool out_used) {
  if (!g) return fail(GSQ_EINVAL, "the sizes are NULL");
  if (!sixteen_bits(g->dtype)) return fail(GSQ_EINVAL, "dtype must be BF16 or FP16, got %d", g->dtype);
  gsq_status st = check_features("in_features", g->in_features);
  if (st == GSQ_OK && out_used) st = check_features("out_features", g->out_features);
  return st == GSQ_OK ? check_sizes(g->groups, g->rows, offsets) : st;
}

gsq::ProductArgs product_args(const gsq_grouped* g, const int64_t* offsets, const void* a, const void* b,
                              void* out, int32_t out_dtype) {
  gsq::ProductArgs p{};
  p.rows = {offsets, g->rows, g->groups};
  p.a = a;
  p.b = b;
  p.out = out;
  p.O = g->out_features;
  p.I = g->in_features;
  p.out_dtype = out_dtype;
  return p;
}

void free_linear(gsq_linear* h, bool idle) {
  const size_t limit = idle ? gsq::DevicePool::limit() : 0;
  for (int i = 0; i < h->n_bufs; ++i) {
    if (idle)
      gsq::g_pool.give(h->device, h->bufs[i].p, h->bufs[i].bytes, limit);
    else
      (void)hipFree(h->bufs[i].p);
  }
  delete h;
}

}  // namespace

extern "C" {

gsq_status gsq_grouped_forward(const gsq_grouped* g, const void* x, const void* w,
                               const int64_t* offsets, void* y, hipStream_t stream) {
  gsq::clear_error();
  GSQ_TRY(check_grouped(g, offsets, true));
  GSQ_TRY(check_array("x", x, 2, g->rows > 0));
  GSQ_TRY(check_array("w", w, 2, true));
  GSQ_TRY(check_array("y", y, 2, g->rows > 0));
  return launched(gsq::launch_product(gsq::kForward, g->dtype, product_args(g, offsets, x, w, y, g->dtype), stream),
                  "gsq_grouped_forward");
}

gsq_status gsq_grouped_input_grad(const gsq_grouped* g, const void* dy, const void* w,
                                  const int64_t* offsets, void* dx, hipStream_t stream) {
  gsq::clear_error();
  GSQ_TRY(check_grouped(g, offsets, true));
  GSQ_TRY(check_array("dy", dy, 2, g->rows > 0));
  GSQ_TRY(check_array("w", w, 2, true));
  GSQ_TRY(check_array("dx", dx, 2, g->rows > 0));
  return launched(gsq::launch_product(gsq::kInputGrad, g->dtype, product_args(g, offsets, dy, w, dx, g->dtype), stream),
                  "gsq_grouped_input_grad");
}

gsq_status gsq_grouped_weight_grad(const gsq_grouped* g, const void* dy, const void* x,
                                   const int64_t* offsets, void* dw, int32_t dw_dtype,
                                   int32_t accumulate, hipStream_t stream) {
  gsq::clear_error();
  GSQ_TRY(check_grouped(g, offsets, true));
  if (dw_dtype != g->dtype && dw_dtype != GSQ_DT_FP32)
    return fail(GSQ_EINVAL, "dw_dtype must be the type of x or FP32, got %d", dw_dtype);
  if (accumulate && dw_dtype != GSQ_DT_FP32)
    return fail(GSQ_EINVAL, "gradients accumulate in FP32 only");
  GSQ_TRY(check_array("dy", dy, 2, g->rows > 0));
  GSQ_TRY(check_array("x", x, 2, g->rows > 0));
  GSQ_TRY(check_array("dw", dw, dw_dtype == GSQ_DT_FP32 ? 4 : 2, true));
  gsq::ProductArgs p = product_args(g, offsets, dy, x, dw, dw_dtype);
  p.accumulate = accumulate ? 1 : 0;
  return launched(gsq::launch_product(gsq::kWeightGrad, g->dtype, p, stream),
                  "gsq_grouped_weight_grad");
}

gsq_status gsq_gram(const gsq_grouped* g, const void* x, const int64_t* offsets, float* h,
                    int32_t accumulate, hipStream_t stream) {
  gsq::clear_error();
  GSQ_TRY(check_grouped(g, offsets, false));
  GSQ_TRY(check_array("x", x, 2, g->rows > 0));
  GSQ_TRY(check_array("h", h, 4, true));
  gsq::ProductArgs p = product_args(g, offsets, x, x, h, GSQ_DT_FP32);
  p.O = g->in_features;
  p.accumulate = accumulate ? 1 : 0;
  return launched(gsq::launch_gram(g->dtype, p, stream),
                  "gsq_gram");
}

gsq_status gsq_quantize_rows(const void* x, int32_t dtype, int64_t rows, int32_t cols, int8_t* q,
                             float* scales, hipStream_t stream) {
  gsq::clear_error();
  if (!sixteen_bits(dtype) && dtype != GSQ_DT_FP32) return fail(GSQ_EINVAL, "unknown dtype %d", dtype);
  if (rows < 0 || rows > (1 << 23))
    return fail(GSQ_EINVAL, "rows must be in [0, 8388608], got %lld", (long long)rows);
  GSQ_TRY(check_features("cols", cols));
  GSQ_TRY(check_array("x", x, dtype == GSQ_DT_FP32 ? 4 : 2, rows > 0));
  GSQ_TRY(check_array("q", q, 1, rows > 0));
  GSQ_TRY(check_array("scales", scales, 4, rows > 0));
  GSQ_HIP(gsq::launch_quantize_rows(x, dtype, rows, cols, q, scales, stream));
  return GSQ_OK;
}

gsq_status gsq_grouped_forward_i8(const gsq_grouped* g, const int8_t* x, const float* x_scales,
                                  const int8_t* w, const float* w_scales, const int64_t* offsets,
                                  void* y, hipStream_t stream) {
  gsq::clear_error();
  GSQ_TRY(check_grouped(g, offsets, true));
  if (g->in_features > kMostExactI8)
    return fail(GSQ_EINVAL, "in_features must be at most %d for exact 32-bit sums, got %d", kMostExactI8,
                g->in_features);
  GSQ_TRY(check_array("x", x, 1, g->rows > 0));
  GSQ_TRY(check_array("x_scales", x_scales, 4, g->rows > 0));
  GSQ_TRY(check_array("w", w, 1, true));
  GSQ_TRY(check_array("w_scales", w_scales, 4, true));
  GSQ_TRY(check_array("y", y, 2, g->rows > 0));
  gsq::ProductArgs p = product_args(g, offsets, x, w, y, g->dtype);
  p.a_scales = x_scales;
  p.b_scales = w_scales;
  return launched(gsq::launch_product_i8(p, stream),
                  "gsq_grouped_forward_i8");
}

gsq_status gsq_linear_init(const gsq_config* cfg, const void* packed, size_t packed_bytes,
                           hipStream_t stream, gsq_linear** out) {
  gsq::clear_error();
  if (!out) return fail(GSQ_EINVAL, "out is NULL");
  *out = nullptr;
  GSQ_TRY(gsq::validate_config(cfg));
  if (!packed) return fail(GSQ_EINVAL, "packed is NULL");
  const size_t need = gsq_packed_size(cfg);
  if (packed_bytes < need)
    return fail(GSQ_EINVAL, "packed buffer has %zu bytes, needs %zu", packed_bytes, need);
  GSQ_TRY(check_features("in_features", cfg->in_features));
  GSQ_TRY(check_features("out_features", cfg->out_features));
  if (cfg->batch > kMostGroups)
    return fail(GSQ_EINVAL, "batch must be at most %d, got %d", kMostGroups, cfg->batch);
  hipStreamCaptureStatus capture = hipStreamCaptureStatusNone;
  GSQ_HIP(hipStreamIsCapturing(stream, &capture));
  if (capture != hipStreamCaptureStatusNone)
    return fail(GSQ_EINVAL, "gsq_linear_init allocates and cannot be captured");

  gsq_linear* h = new (std::nothrow) gsq_linear{};
  if (!h) return fail(GSQ_ENOMEM, "host allocation failed");
  const bool super = cfg->layout == GSQ_LAYOUT_SUPERBLOCK;
  gsq::PackedLayer& L = h->L;
  L.O = cfg->out_features;
  L.I = cfg->in_features;
  L.gs = super ? 256 : cfg->group_size;
  L.n_levels = cfg->n_levels;
  L.bits = super ? 3 : gsq::code_bits(cfg->n_levels);
  L.tiles = (L.O + 15) / 16;
  L.blocks = (L.I + 127) / 128;
  L.scale_groups = (L.blocks * 128 + L.gs - 1) / L.gs;
  for (int k = 0; k < GSQ_MAX_LEVELS; ++k) L.levels[k] = cfg->levels[k < L.n_levels ? k : L.n_levels - 1];
  h->groups = cfg->batch;
  hipError_t e = hipGetDevice(&h->device);
  if (e != hipSuccess) {
    delete h;
    return gsq::hip_fail(e, "hipGetDevice");
  }
  const gsq::KeptBytes kept = gsq::kept_bytes(cfg->batch, L.O, L.I, L.bits, L.gs, super);
  const size_t bytes[3] = {(size_t)kept.codes, (size_t)kept.scales, (size_t)kept.sub};
  for (int i = 0; i < 3; ++i) {
    if (!bytes[i]) continue;
    void* p = nullptr;
    size_t got = 0;
    if (gsq::g_pool.take(h->device, bytes[i], &p, &got) != hipSuccess) {
      (void)hipGetLastError();
      free_linear(h, true);   // nothing was enqueued
      return fail(GSQ_ENOMEM, "device allocation failed for a packed %d x %d x %d layer", cfg->batch,
                  L.O, L.I);
    }
    h->bufs[h->n_bufs++] = {p, got};
  }
  L.codes = static_cast<const uint32_t*>(h->bufs[0].p);
  L.scales = static_cast<const uint16_t*>(h->bufs[1].p);
  L.sub = super ? static_cast<const uint8_t*>(h->bufs[2].p) : nullptr;
  e = gsq::launch_unpack_layer(*cfg, static_cast<const uint8_t*>(packed), L, stream);
  if (e != hipSuccess) {
    free_linear(h, hipStreamSynchronize(stream) == hipSuccess);
    return gsq::hip_fail(e, "laying out the packed layer");
  }
  *out = h;
  return GSQ_OK;
}

gsq_status gsq_linear_forward(const gsq_linear* h, const void* x, int32_t dtype, int64_t rows,
                              const int64_t* offsets, void* y, hipStream_t stream) {
  gsq::clear_error();
  if (!h) return fail(GSQ_EINVAL, "handle is NULL");
  if (!sixteen_bits(dtype)) return fail(GSQ_EINVAL, "dtype must be BF16 or FP16, got %d", dtype);
  GSQ_TRY(check_sizes(h->groups, rows, offsets));
  GSQ_TRY(check_array("x", x, 2, rows > 0));
  GSQ_TRY(check_array("y", y, 2, rows > 0));
  int dev = -1;
  GSQ_HIP(hipGetDevice(&dev));
  if (dev != h->device)
    return fail(GSQ_EINVAL, "the handle was created on device %d, device %d is current", h->device, dev);
  return launched(gsq::launch_packed_product(h->L, dtype, gsq::GroupRows{offsets, rows, h->groups}, x, y, stream),
                  "gsq_linear_forward");
}

gsq_status gsq_linear_destroy(gsq_linear* h) {
  if (!h) return GSQ_OK;
  // its own device must be idle (and be the current one, as the kept blocks' limit is)
  int dev = -1;
  const int h_device = h->device;
  const bool own = hipGetDevice(&dev) == hipSuccess &&
                   (dev == h_device || hipSetDevice(h_device) == hipSuccess);
  const bool idle = hipDeviceSynchronize() == hipSuccess;
  free_linear(h, own && idle);
  if (own && dev != h_device) (void)hipSetDevice(dev);
  return GSQ_OK;
}

}  // extern "C"
