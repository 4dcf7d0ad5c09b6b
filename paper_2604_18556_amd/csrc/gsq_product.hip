// Products of rows that are grouped by layer (the tokens of each routed expert): the layer's output, the
// gradients of its input and weights, the Gram matrix of its inputs, and the output in 8-bit integers.
#include <hip/hip_runtime.h>

#include <algorithm>

#include "gsq_product_any.hpp"

namespace gsq {
namespace {

// y or dx: a panel of 64 rows of one group times that group's weights.
template <class T, int kForm>
__global__ __launch_bounds__(256) void k_rows_any(ProductArgs p) {
  using E = typename T::elem;
  int e;
  int64_t first, end;
  if (!find_panel(p.rows, kAnyTile, blockIdx.x, e, first, end)) return;
  const int n0 = blockIdx.y * kAnyTile, ms = (int)(end - first);
  const int ks = kForm == kForward ? p.I : p.O, ns = kForm == kForward ? p.O : p.I;
  const E* w = static_cast<const E*>(p.b) + (int64_t)e * p.O * p.I;
  const AlongK<E> a{static_cast<const E*>(p.a) + first * ks, ks, ms, ks};
  const auto store = [&](int m, int n, auto v) {
    if (m >= ms || n >= ns) return;
    float y = (float)v;
    if constexpr (T::kDtype < 0)   // 8-bit integers: the sum is exact in 32 bits
      y = y * p.a_scales[first + m] * p.b_scales[(int64_t)e * p.O + n];
    store_out(p.out, p.out_dtype, (first + m) * ns + n, y);
  };
  if constexpr (kForm == kForward)
    tile_any<T>(a, AlongK<E>{w, p.I, ns, ks}, 0, n0, ks, store);
  else
    tile_any<T>(a, AcrossK<E>{w, p.I, ns, ks}, 0, n0, ks, store);
}

// dW of one group (blockIdx.z): the sum runs over the group's rows; without rows it is zero.
template <class T>
__global__ __launch_bounds__(256) void k_weight_grad_any(ProductArgs p) {
  using E = typename T::elem;
  const int e = blockIdx.z;
  int64_t first, end;
  group_rows(p.rows, e, first, end);
  const int ks = (int)(end - first);
  const AcrossK<E> a{static_cast<const E*>(p.a) + first * p.O, p.O, p.O, ks};
  const AcrossK<E> b{static_cast<const E*>(p.b) + first * p.I, p.I, p.I, ks};
  const auto store = [&](int m, int n, float v) {
    if (m >= p.O || n >= p.I) return;
    const int64_t at = ((int64_t)e * p.O + m) * p.I + n;
    if (p.accumulate) v += static_cast<const float*>(p.out)[at];
    store_out(p.out, p.out_dtype, at, v);
  };
  tile_any<T>(a, b, blockIdx.y * kAnyTile, blockIdx.x * kAnyTile, ks, store);
}

// Rows in 8-bit integers: s = max |x| / 127 in fp32, q = x / s to the nearest integer, ties to even.  A
// row of zeros has s = 0 and q = 0; a row with an infinity or NaN s = NaN and q = 0, so that its products
// are NaN.
template <class E>
__global__ __launch_bounds__(256) void k_quantize_rows(const E* __restrict__ x, int64_t cols,
                                                       int8_t* __restrict__ q, float* __restrict__ scales) {
  __shared__ float part[4];
  __shared__ int bad_part[4];
  const int64_t row = blockIdx.x;
  x += row * cols;
  q += row * cols;
  float top = 0.f;
  bool bad = false;
  for (int64_t c = threadIdx.x; c < cols; c += 256) {
    const float v = fabsf((float)x[c]);
    bad |= !(v <= __FLT_MAX__);
    top = fmaxf(top, v);
  }
#pragma unroll
  for (int d = 32; d; d >>= 1) top = fmaxf(top, __shfl_xor(top, d, 64));
  const bool wave_bad = __any(bad);
  if ((threadIdx.x & 63) == 0) {
    part[threadIdx.x >> 6] = top;
    bad_part[threadIdx.x >> 6] = wave_bad;
  }
  __syncthreads();
  top = fmaxf(fmaxf(part[0], part[1]), fmaxf(part[2], part[3]));
  bad = bad_part[0] | bad_part[1] | bad_part[2] | bad_part[3];
  const float s = bad ? __builtin_nanf("") : top / 127.f;
  if (threadIdx.x == 0) scales[row] = s;
  for (int64_t c = threadIdx.x; c < cols; c += 256) {
    const float v = (float)x[c];
    float r = 0.f;
    if (s > 0.f) {
      // the division may round onto a half, or off it: the remainder, exact in an fma, decides
      r = rintf(v / s);
      const float rest = fmaf(-r, s, v), twice = 2.f * fabsf(rest);
      if (twice > s || (twice == s && ((int)r & 1))) r += copysignf(1.f, rest);
      r = fminf(fmaxf(r, -127.f), 127.f);
    }
    q[c] = (int8_t)r;
  }
}

}  // namespace

hipError_t launch_product(int form, int dtype, const ProductArgs& p, hipStream_t s) {
  if (form == kWeightGrad) {
    const dim3 grid((p.I + kAnyTile - 1) / kAnyTile, (p.O + kAnyTile - 1) / kAnyTile, p.rows.groups);
    if (dtype == GSQ_DT_BF16)
      k_weight_grad_any<Bf16><<<grid, 256, 0, s>>>(p);
    else
      k_weight_grad_any<F16><<<grid, 256, 0, s>>>(p);
    return hipGetLastError();
  }
  if (p.rows.rows == 0) return hipSuccess;
  const int ns = form == kForward ? p.O : p.I;
  const dim3 grid(most_panels(p.rows, kAnyTile), (ns + kAnyTile - 1) / kAnyTile);
  if (form == kForward && dtype == GSQ_DT_BF16)
    k_rows_any<Bf16, kForward><<<grid, 256, 0, s>>>(p);
  else if (form == kForward)
    k_rows_any<F16, kForward><<<grid, 256, 0, s>>>(p);
  else if (dtype == GSQ_DT_BF16)
    k_rows_any<Bf16, kInputGrad><<<grid, 256, 0, s>>>(p);
  else
    k_rows_any<F16, kInputGrad><<<grid, 256, 0, s>>>(p);
  return hipGetLastError();
}

hipError_t launch_product_i8(const ProductArgs& p, hipStream_t s) {
  if (p.rows.rows == 0) return hipSuccess;
  const dim3 grid(most_panels(p.rows, kAnyTile), (p.O + kAnyTile - 1) / kAnyTile);
  k_rows_any<I8, kForward><<<grid, 256, 0, s>>>(p);
  return hipGetLastError();
}

hipError_t launch_gram(int dtype, const ProductArgs& p, hipStream_t s) {
  return launch_product(kWeightGrad, dtype, p, s);
}

hipError_t launch_quantize_rows(const void* x, int dtype, int64_t rows, int64_t cols, int8_t* q,
                                float* scales, hipStream_t s) {
  if (rows == 0) return hipSuccess;
  if (dtype == GSQ_DT_BF16)
    k_quantize_rows<<<rows, 256, 0, s>>>(static_cast<const __bf16*>(x), cols, q, scales);
  else if (dtype == GSQ_DT_FP16)
    k_quantize_rows<<<rows, 256, 0, s>>>(static_cast<const _Float16*>(x), cols, q, scales);
  else
    k_quantize_rows<<<rows, 256, 0, s>>>(static_cast<const float*>(x), cols, q, scales);
  return hipGetLastError();
}

}  // namespace gsq
