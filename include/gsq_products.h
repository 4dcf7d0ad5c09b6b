/*
 * gsq_products.h -- the products around the layer's optimisation, in the same library as gsq.h.
 *
 * The matrix products that a user of the step needs beside it: H before it, the layer's output and its
 * gradients with the dense weights, and the output with the packed codes or with 8-bit integers after
 * it.  Rows (tokens) of all groups (the layers of a batch: routed experts) come together, sorted by
 * group.  `offsets` is a device array of groups + 1 int64: group e has the rows offsets[e] ..
 * offsets[e + 1] - 1, possibly none; NULL means that every row belongs to the one group.  The host never
 * reads it, so the calls can be captured into a HIP graph and replayed with other offsets.  Offsets have
 * to be in [0, rows] and must not fall.  Others are read as the nearest that do, and give unspecified
 * values inside the outputs.  Output rows of no group are left as they were.
 *
 * Stream, device pointers, status codes and gsq_last_error() are as gsq.h says; every array is dense and
 * row-major.  These calls allocate nothing, synchronise nothing and keep no scratch.  Any number of them may run at
 * once, on any streams, as long as their outputs do not overlap.  An output must not overlap an input.
 * Sums are held in fp32 (int32 for 8-bit integers) in a fixed order: equal inputs give equal bits on the
 * same device, though not between the two sides of a size rule.  Infinities and NaN go through as the
 * arithmetic has them, within the rows and channels they belong to.  Pointers need the alignment of their
 * elements only; arrays with 16-byte aligned bases and rows are read faster.  Limits (GSQ_EINVAL):
 * groups <= 65535, rows <= 2^29, out_features and in_features <= 2^21, and the tiles of one launch.  Those
 * are never too many while (rows / 64 + min(rows, groups)) ceil(n / 64) < 2^23, n being the columns of the
 * output, or for sums over rows (dW, H) groups ceil(O / 64) ceil(I / 64) < 2^23.  The device that the
 * pointers belong to has to be current.
 */
#ifndef GSQ_PRODUCTS_H
#define GSQ_PRODUCTS_H

#include "gsq.h"

#ifdef __cplusplus
extern "C" {
#endif

enum { GSQ_DT_FP16 = 2 };   /* beside GSQ_DT_FP32 and GSQ_DT_BF16 */

typedef struct {
  int32_t groups;          /* layers: w holds one O x I matrix for each (>= 1)                 */
  int32_t out_features;    /* O (>= 1)                                                         */
  int32_t in_features;     /* I (>= 1)                                                         */
  int32_t dtype;           /* GSQ_DT_BF16 or GSQ_DT_FP16: x, w, y and their gradients          */
  int64_t rows;            /* R: rows of x and y, of all groups together (>= 0)                */
} gsq_grouped;

/* y = x W_e^T.  x: R x I, w: groups x O x I, y: R x O, each value rounded once. */
gsq_status gsq_grouped_forward(const gsq_grouped* g, const void* x, const void* w,
                               const int64_t* offsets, void* y, hipStream_t stream);

/* The gradient of x: dx = dy W_e.  dy: R x O, w: groups x O x I, dx: R x I. */
gsq_status gsq_grouped_input_grad(const gsq_grouped* g, const void* dy, const void* w,
                                  const int64_t* offsets, void* dx, hipStream_t stream);

/* The gradient of W: dW_e = sum over the rows r of e of dy[r]^T x[r].  dy: R x O, x: R x I, dw: groups x
 * O x I in dw_dtype, which is dtype or GSQ_DT_FP32.  A group without rows gets zeros.  accumulate != 0
 * adds to what dw holds (fp32 only: 16 bits would lose small batches). */
gsq_status gsq_grouped_weight_grad(const gsq_grouped* g, const void* dy, const void* x,
                                   const int64_t* offsets, void* dw, int32_t dw_dtype,
                                   int32_t accumulate, hipStream_t stream);

/* H_e = X_e^T X_e, what gsq_layer_init takes: x: R x I, h: fp32 groups x I x I, exactly symmetric (as
 * far as h was, when it accumulates).  accumulate != 0 adds to h, one calibration batch after another.
 * out_features is not used. */
gsq_status gsq_gram(const gsq_grouped* g, const void* x, const int64_t* offsets, float* h,
                    int32_t accumulate, hipStream_t stream);

/* Rows in 8-bit integers: scales[r] = max |x[r]| / 127 (fp32), q = x / scale to the nearest integer, ties
 * to even, of the exact quotient, within [-127, 127].  x: rows x cols in dtype (GSQ_DT_*), q: int8 rows x
 * cols, scales: fp32 rows.  A row of zeros has scale 0 and q = 0.  A row with an infinity or NaN has scale
 * NaN and q = 0, so that what is computed from it is NaN.  Tokens are rows of x; a layer's output channels
 * are the rows of its weights.  rows <= 2^23, cols <= 2^21. */
gsq_status gsq_quantize_rows(const void* x, int32_t dtype, int64_t rows, int32_t cols, int8_t* q,
                             float* scales, hipStream_t stream);

/* y[r, n] = x_scales[r] w_scales[e, n] sum_k x[r, k] w[e, n, k] for 8-bit x and w.  x: int8 R x I, x_scales:
 * fp32 R, w: int8 groups x O x I, w_scales: fp32 groups x O, y: R x O in dtype.  The sum is exact:
 * in_features <= 131071.  It is then scaled in fp32, by x's scale first: (sum x_scale) w_scale. */
gsq_status gsq_grouped_forward_i8(const gsq_grouped* g, const int8_t* x, const float* x_scales,
                                  const int8_t* w, const float* w_scales, const int64_t* offsets,
                                  void* y, hipStream_t stream);

/*
 * A packed layer in use.  gsq_linear_init reads the bytes that gsq_pack wrote for cfg (batch, sizes,
 * levels, group_size and layout count) and lays them out for the matrix cores, in units of 16 channels x
 * 128 inputs.  It keeps the packed bytes of the layer with its sizes rounded up to those, and a quarter
 * more at most (1.6-bit codes take 2 bits, 6-bit scales 8): a layer of few channels or inputs takes a
 * multiple of its own.  `packed` may be freed once the stream has passed the call.  A code >= n_levels is
 * read as n_levels - 1.  It allocates, so a capturing stream is refused.
 *
 * gsq_linear_forward: y = x Wq_e^T for x: rows x I and y: rows x O in dtype (GSQ_DT_BF16 or GSQ_DT_FP16),
 * rows grouped by the layers of the batch.  A weight is scale * level in fp32 (SUPERBLOCK: d * sc * level,
 * d * sc being exact), rounded to dtype: the values that a 16-bit copy of the layer would hold.  Sums are
 * in fp32.  The handle is read only: calls on one handle may overlap on several streams, once the stream of
 * gsq_linear_init has passed that call.  It works on the device it was made on, which has to be current.
 *
 * gsq_linear_destroy: NULL-safe; synchronises the device.  The buffers are kept or freed as those of a
 * gsq_layer are.
 */
typedef struct gsq_linear gsq_linear;

gsq_status gsq_linear_init(const gsq_config* cfg, const void* packed, size_t packed_bytes,
                           hipStream_t stream, gsq_linear** out);
gsq_status gsq_linear_forward(const gsq_linear* h, const void* x, int32_t dtype, int64_t rows,
                              const int64_t* offsets, void* y, hipStream_t stream);
gsq_status gsq_linear_destroy(gsq_linear* h);

#ifdef __cplusplus
}
#endif

#endif /* GSQ_PRODUCTS_H */
