// Internal declarations of the products of grouped rows and of the packed layer.
#pragma once
#include <hip/hip_runtime.h>
#include <stdint.h>

#include "gsq_products.h"

namespace gsq {

// Rows of all groups together, sorted by group: group e has the rows offsets[e] .. offsets[e + 1] - 1
// (NULL: one group, all rows).
struct GroupRows {
  const int64_t* offsets;
  int64_t rows;
  int32_t groups;
};

enum { kForward = 0, kInputGrad = 1, kWeightGrad = 2 };

// One product.  kForward: out[r, n] = sum_k a[r, k] b[e][n, k]; kInputGrad: out[r, k] = sum_n a[r, n]
// b[e][n, k]; kWeightGrad: out[e][n, k] = sum_r a[r, n] b[r, k].
struct ProductArgs {
  GroupRows rows;
  const void* a;
  const void* b;
  void* out;
  int32_t O, I;
  int32_t out_dtype;          // GSQ_DT_*
  int32_t height;             // of a panel of rows
  int32_t vector_out;         // results may be stored four at a time
  int32_t accumulate;         // kWeightGrad into fp32: add to what is there
  const float* a_scales;      // 8-bit integers: one per row, and one per group and channel
  const float* b_scales;
};

// A packed layer as the kernels read it.  Weights come in units of 16 output channels x 128 inputs:
// lane l = 16 g + n of a wavefront has the 32 codes of channel n at inputs 32 g .. 32 g + 31, `bits`
// 32-bit words of them (word_of_codes).  Channels beyond O and inputs beyond I have scale zero.
struct PackedLayer {
  const uint32_t* codes;      // groups x tiles x blocks x 64 lanes x bits
  const uint16_t* scales;     // fp16 (SUPERBLOCK: d): groups x tiles x scale groups x 16 channels, or for
                              // groups of 16 inputs, two for each lane of each unit
  const uint8_t* sub;         // SUPERBLOCK: the 6-bit scales, two for each lane of each unit; else NULL
  int32_t O, I, bits, gs;     // gs: inputs per fp16 scale
  int32_t tiles, blocks;      // of 16 channels, of 128 inputs
  int32_t scale_groups;       // per channel
  int32_t n_levels;
  float levels[GSQ_MAX_LEVELS];   // those past n_levels repeat the last
};

hipError_t launch_product(int form, int dtype, const ProductArgs& p, hipStream_t s);
hipError_t launch_product_i8(const ProductArgs& p, hipStream_t s);
hipError_t launch_gram(int dtype, const ProductArgs& p, hipStream_t s);
hipError_t launch_quantize_rows(const void* x, int dtype, int64_t rows, int64_t cols, int8_t* q,
                                float* scales, hipStream_t s);
hipError_t launch_unpack_layer(const gsq_config& cfg, const uint8_t* packed, const PackedLayer& L,
                               hipStream_t s);
hipError_t launch_packed_product(const PackedLayer& L, int dtype, const GroupRows& rows, const void* x,
                                 void* y, hipStream_t s);

}  // namespace gsq
