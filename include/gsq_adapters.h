/*
 * gsq_adapters.h -- low-rank adapters of many requests beside a shared projection, in the same library as gsq.h.
 *
 * Rows (tokens) come together request by request: segment i has the rows offsets[i] .. offsets[i + 1] - 1 (NULL:
 * one segment has all), read as gsq_products.h says, and the adapter index[i], another than 0 .. adapters - 1 (-1)
 * being none; several segments may have the same adapter.  index NULL means that segment i has adapter i
 * (adapters == segments).  The projection itself is a product of gsq_products.h, dense, packed or in 8 bits; its
 * output or input gradient comes as `base`, to which the adapters' part is added, and may be NULL (zeros) or the
 * output itself (in place).  With A: adapters x rank x I, B: adapters x O x rank, scales: fp32 per adapter or NULL
 * (ones), and e the adapter of row r:
 *
 *   forward      hidden[r] = A_e x[r]                    y[r]  = base[r] + scale_e B_e hidden[r]
 *   input grad   dhidden[r] = scale_e B_e^T dy[r]        dx[r] = base[r] + A_e^T dhidden[r]
 *   weight grad  dA_e = sum_r dhidden[r]^T x[r]          dB_e = scale_e sum_r dy[r]^T hidden[r]
 *
 * hidden and dhidden (fp32 R x rank) are outputs of the first two and inputs of the third.  Rows of segments
 * without an adapter get hidden 0 and y = base; rows of no segment are left as they were.  An adapter of a lower
 * rank is padded with zeros.
 *
 * Stream, device pointers, status codes and gsq_last_error() are as gsq.h says, addresses, overlapping calls and
 * reproducibility as gsq_products.h does; nothing is allocated, synchronised or kept.  Sums are in fp32, and y and dx
 * are rounded once: hidden enters the second product off by no more than 2^-16 of each value (bf16), or by 2^-22 of it
 * and 2^-36 of the row's largest (fp16).  What is not finite stays in its rows of y and dx, and in its adapter's
 * gradients; where the formulas have an infinity there may be NaN.
 */
#ifndef GSQ_ADAPTERS_H
#define GSQ_ADAPTERS_H

#include "gsq_products.h"

#ifdef __cplusplus
extern "C" {
#endif

#define GSQ_MAX_RANK 512

typedef struct {
  int32_t segments;        /* rows of one adapter each (1 .. 65535)                               */
  int32_t adapters;        /* (1 .. 65535)                                                        */
  int32_t rank;            /* (1 .. GSQ_MAX_RANK)                                                 */
  int32_t out_features;    /* O (1 .. 2^21)                                                       */
  int32_t in_features;     /* I (1 .. 2^21)                                                       */
  int32_t dtype;           /* of x, y, A, B and base: GSQ_DT_BF16 or GSQ_DT_FP16                  */
  int64_t rows;            /* R: rows of x and y, of all segments together (0 .. 2^29)            */
} gsq_adapters;

/* x: R x I, base, y: R x O, hidden: fp32 R x rank. */
gsq_status gsq_adapter_forward(const gsq_adapters* g, const void* x, const void* a, const void* b,
                               const int64_t* offsets, const int32_t* index, const float* scales,
                               const void* base, float* hidden, void* y, hipStream_t stream);

/* dy: R x O, base, dx: R x I, dhidden: fp32 R x rank. */
gsq_status gsq_adapter_input_grad(const gsq_adapters* g, const void* dy, const void* a, const void* b,
                                  const int64_t* offsets, const int32_t* index, const float* scales,
                                  const void* base, float* dhidden, void* dx, hipStream_t stream);

/* da: adapters x rank x I, db: adapters x O x rank, both in dw_dtype, which is dtype or GSQ_DT_FP32.  An adapter
 * without rows gets zeros.  accumulate != 0 adds to what da and db hold (fp32 only). */
gsq_status gsq_adapter_weight_grad(const gsq_adapters* g, const void* dy, const void* x, const float* hidden,
                                   const float* dhidden, const int64_t* offsets, const int32_t* index,
                                   const float* scales, void* da, void* db, int32_t dw_dtype,
                                   int32_t accumulate, hipStream_t stream);

#ifdef __cplusplus
}
#endif

#endif /* GSQ_ADAPTERS_H */
