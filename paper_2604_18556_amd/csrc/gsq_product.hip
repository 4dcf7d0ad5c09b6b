// Products of rows that are grouped by layer (the tokens of each routed expert): the layer's output, the
// gradients of its input and weights, the Gram matrix of its inputs, and the output in 8-bit integers.
#include <hip/hip_runtime.h>

#include <algorithm>

#include "gsq_tile.hpp"

namespace gsq {
namespace {

// y or dx: a panel of 64 rows of one group times that group's weights.
template <class T, int kForm>
__global__ __launch_bounds__(256) void k_rows_any(ProductArgs p) {
  using E = typename T::elem;
  PanelPlace at;
  if (!find_panel(p.rows, kAnyTile, blockIdx.x, at)) return;
  const int64_t first = at.first + (int64_t)at.panel * kAnyTile;
  const int e = at.group, ms = (int)min(at.end - first, (int64_t)kAnyTile);
  const int n0 = blockIdx.y * kAnyTile;
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

// One tile of y or dx: rows m0 .. of a group, columns n0 .. .
template <class T, int kForm, class S>
__device__ __forceinline__ void rows_tile(const ProductArgs& p, const RowsTile& at, uint8_t* smem) {
  const int64_t first = at.first;
  const int ms = at.ms, n0 = at.n0;
  using E = typename T::elem;
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int ks = kForm == kForward ? p.I : p.O, ns = kForm == kForward ? p.O : p.I;
  const int nk = (int)(((int64_t)ks * sizeof(E) + ROW_BYTES - 1) / ROW_BYTES);
  const E* w = static_cast<const E*>(p.b) + (int64_t)at.group * p.O * p.I;
  const SlabAlong<S::TM> a(static_cast<const E*>(p.a) + first * ks, (int64_t)ks * sizeof(E), ms, wave, lane);
  typename T::acc acc[S::MI][S::NJ];
  if constexpr (kForm == kForward) {
    SlabAlong<S::TN> b(w + (int64_t)n0 * ks, (int64_t)ks * sizeof(E), ns - n0, wave, lane);
    tile_ring<T, S>(a, b, nk, acc, smem);
  } else {
    SlabAcross<S::TN> b(w + n0, (int64_t)ns * sizeof(E), ns - n0, ks, wave, lane);
    tile_ring<T, S>(a, b, nk, acc, smem);
  }
  const bool four = p.vector_out;
  tile_results<S>(acc, [&](int m, int n, auto v) {
    if (m >= ms || n0 + n >= ns) return;
    f32x4 y;
#pragma unroll
    for (int c = 0; c < 4; ++c) y[c] = (float)v[c];
    if constexpr (T::kDtype < 0) {   // 8-bit integers: the sum is exact in 32 bits
      const float* bs = p.b_scales + (int64_t)at.group * p.O + n0 + n;
      const float as = p.a_scales[first + m];
#pragma unroll
      for (int c = 0; c < 4; ++c) y[c] = y[c] * as * bs[min(c, ns - n0 - n - 1)];
    }
    store_four(p.out, p.out_dtype, (first + m) * ns + n0 + n, y, ns - n0 - n, four);
  });
}

// y or dx.
template <class T, int kForm>
__global__ __launch_bounds__(256, 1) void k_rows_tile(ProductArgs p) {
  extern __shared__ __attribute__((aligned(16))) uint8_t smem[];
  RowsTile at;
  if (!find_rows_tile(p.rows, p.height, kForm == kForward ? p.O : p.I, at)) return;
  if (at.ms > Half::TM)
    rows_tile<T, kForm, Whole>(p, at, smem);
  else if (at.ms > Low::TM)
    rows_tile<T, kForm, Half>(p, at, smem);
  else
    rows_tile<T, kForm, Low>(p, at, smem);
}

// One tile of a sum over a group's rows: out[m0 .., n0 ..] (+)= sum_r a[r, m] b[r, n], and with `mirror` its
// transpose too.
template <class T>
__device__ __forceinline__ void sum_tile(const ProductArgs& p, int e, int m0, int n0, bool mirror, uint8_t* smem) {
  using E = typename T::elem;
  using S = Whole;
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  int64_t first, end;
  group_rows(p.rows, e, first, end);
  const int ks = (int)(end - first), nk = (ks + kSlabRows - 1) / kSlabRows;
  // a group without rows reads zeros only: its addresses are not used
  const SlabAcross<S::TM> a(static_cast<const E*>(p.a) + first * p.O + m0, (int64_t)p.O * 2, p.O - m0, ks, wave, lane);
  SlabAcross<S::TN> b(static_cast<const E*>(p.b) + first * p.I + n0, (int64_t)p.I * 2, p.I - n0, ks, wave, lane);
  typename T::acc acc[S::MI][S::NJ];
  tile_ring<T, S>(a, b, nk, acc, smem);
  const int64_t out0 = (int64_t)e * p.O * p.I;
  tile_results<S>(acc, [&](int m, int n, f32x4 v) {
    m += m0;
    n += n0;
    if (m >= p.O || n >= p.I) return;
    const int64_t at = out0 + (int64_t)m * p.I + n;
    if (p.accumulate) {
      const float* sums = static_cast<const float*>(p.out) + at;
#pragma unroll
      for (int c = 0; c < 4; ++c) v[c] += n + c < p.I ? sums[c] : 0.f;
    }
    store_four(p.out, p.out_dtype, at, v, p.I - n, p.vector_out);
  });
  if (!mirror) return;
  tile_results<S>(acc, [&](int m, int n, f32x4 v) {   // 16 lanes hold 16 neighbours of a transposed row
    m += m0;
    n += n0;
    if (m >= p.O) return;
    float* sums = static_cast<float*>(p.out) + out0 + (int64_t)n * p.I + m;
#pragma unroll
    for (int c = 0; c < 4; ++c, sums += p.I)
      if (n + c < p.I) *sums = p.accumulate ? *sums + v[c] : v[c];
  });
}

// dW of every group, each group's tiles spread over the XCDs.
template <class T>
__global__ __launch_bounds__(256, 1) void k_weight_grad_tile(ProductArgs p) {
  extern __shared__ __attribute__((aligned(16))) uint8_t smem[];
  const int tiles_m = (p.O + Whole::TM - 1) / Whole::TM, tiles_n = (p.I + Whole::TN - 1) / Whole::TN;
  const int tiles = tiles_m * tiles_n, e = blockIdx.x / (unsigned)tiles;
  int tm, tn;
  tile_at(lin_of(blockIdx.x - e * tiles, tiles), tiles_m, tiles_n, tm, tn);
  sum_tile<T>(p, e, tm * Whole::TM, tn * Whole::TN, false, smem);
}

// H of every group: the tiles on and above the diagonal, and their transposes.  Of T tile rows, row r (T - r
// tiles) and row T - 1 - r (r + 1) are taken as one row of T + 1, so that the order of a rectangle serves;
// an odd T's middle row has the second half of its own empty.
template <class T>
__global__ __launch_bounds__(256, 1) void k_gram_tile(ProductArgs p) {
  extern __shared__ __attribute__((aligned(16))) uint8_t smem[];
  const int side = (p.I + Whole::TM - 1) / Whole::TM, pairs = (side + 1) / 2;
  const int tiles = pairs * (side + 1), e = blockIdx.x / (unsigned)tiles;
  int r, c;
  tile_at(lin_of(blockIdx.x - e * tiles, tiles), pairs, side + 1, r, c);
  int tm = r, tn = r + c;
  if (c >= side - r) {
    tm = side - 1 - r;
    tn = tm + c - (side - r);
    if (tm == r) return;
  }
  sum_tile<T>(p, e, tm * Whole::TM, tn * Whole::TN, tm != tn, smem);
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

template <class T, int kForm>
hipError_t launch_rows(ProductArgs p, hipStream_t s) {
  if (p.rows.rows == 0) return hipSuccess;
  const int ns = kForm == kForward ? p.O : p.I;
  const int64_t unit = 16 / (int64_t)sizeof(typename T::elem);
  if (p.O % (kForm == kForward ? 1 : unit) == 0 && p.I % unit == 0 && aligned16(p.a) && aligned16(p.b)) {
    p.vector_out = four_at_once(p.out, p.out_dtype, ns);
    p.height = pick_height(p.rows, ns);
    return launch_ring(k_rows_tile<T, kForm>, most_panels(p.rows, p.height) * tiles_of(ns, Whole::TN), s, p);
  }
  const dim3 grid(most_panels(p.rows, kAnyTile), tiles_of(ns, kAnyTile));
  k_rows_any<T, kForm><<<grid, 256, 0, s>>>(p);
  return hipGetLastError();
}

template <class T>
hipError_t launch_sums(ProductArgs p, bool gram, hipStream_t s) {
  if (p.O % 8 == 0 && p.I % 8 == 0 && aligned16(p.a) && aligned16(p.b)) {
    p.vector_out = four_at_once(p.out, p.out_dtype, p.I);
    const int64_t tm = tiles_of(p.O, Whole::TM), tn = tiles_of(p.I, Whole::TN);
    if (gram) return launch_ring(k_gram_tile<T>, p.rows.groups * ((tn + 1) / 2 * (tn + 1)), s, p);
    return launch_ring(k_weight_grad_tile<T>, p.rows.groups * tm * tn, s, p);
  }
  const dim3 grid(tiles_of(p.I, kAnyTile), tiles_of(p.O, kAnyTile), p.rows.groups);
  k_weight_grad_any<T><<<grid, 256, 0, s>>>(p);
  return hipGetLastError();
}

}  // namespace

hipError_t launch_product(int form, int dtype, const ProductArgs& p, hipStream_t s) {
  const bool bf16 = dtype == GSQ_DT_BF16;
  if (form == kForward) return bf16 ? launch_rows<Bf16, kForward>(p, s) : launch_rows<F16, kForward>(p, s);
  if (form == kInputGrad) return bf16 ? launch_rows<Bf16, kInputGrad>(p, s) : launch_rows<F16, kInputGrad>(p, s);
  return bf16 ? launch_sums<Bf16>(p, false, s) : launch_sums<F16>(p, false, s);
}

hipError_t launch_product_i8(const ProductArgs& p, hipStream_t s) { return launch_rows<I8, kForward>(p, s); }

hipError_t launch_gram(int dtype, const ProductArgs& p, hipStream_t s) {
  return dtype == GSQ_DT_BF16 ? launch_sums<Bf16>(p, true, s) : launch_sums<F16>(p, true, s);
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
