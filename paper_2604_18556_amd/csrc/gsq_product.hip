// Products of rows that are grouped by layer (the tokens of each routed expert): the layer's output, the
// gradients of its input and weights, the Gram matrix of its inputs, and the output in 8-bit integers.
#include <hip/hip_runtime.h>

#include <algorithm>

#include "gsq_split.hpp"

namespace gsq {
namespace {

// Four consecutive results of row `first` + m of y or dx from column n, those in bounds.
template <class T>
__device__ __forceinline__ void store_rows(const ProductArgs& p, int group, int64_t first, int ms, int ns, int m,
                                           int n, typename T::acc v) {
  if (m >= ms || n >= ns) return;
  f32x4 y;
#pragma unroll
  for (int c = 0; c < 4; ++c) y[c] = (float)v[c];
  if constexpr (T::kDtype < 0) {   // 8-bit integers: the sum is exact in 32 bits
    const float* bs = p.b_scales + (int64_t)group * p.O + n;
    const float as = p.a_scales[first + m];
#pragma unroll
    for (int c = 0; c < 4; ++c) y[c] = y[c] * as * bs[min(c, ns - n - 1)];
  }
  store_four(p.out, p.out_dtype, (first + m) * ns + n, y, ns - n, p.vector_out);
}

// One tile of y or dx.
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
  tile_results<S>(acc, [&](int m, int n, auto v) { store_rows<T>(p, at.group, first, ms, ns, m, n0 + n, v); });
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

// The same from small tiles: panels of TM rows (of which one of 16 or fewer is taken as 16), TN columns.
template <class T, int kForm, int TM, int TN, bool kLoose>
__device__ __forceinline__ void rows_split(const ProductArgs& p, int group, int64_t first, int ms, int n0,
                                           uint8_t* smem) {
  using E = typename T::elem;
  const int lane = threadIdx.x & 63;
  const int ks = kForm == kForward ? p.I : p.O, ns = kForm == kForward ? p.O : p.I;
  const int nk = (int)(((int64_t)ks * sizeof(E) + ROW_BYTES - 1) / ROW_BYTES);
  const E* w = static_cast<const E*>(p.b) + (int64_t)group * p.O * p.I;
  const E* x = static_cast<const E*>(p.a) + first * ks;
  const auto store = [&](int m, int n, typename T::acc v) { store_rows<T>(p, group, first, ms, ns, m, n0 + n, v); };
  if constexpr (kLoose) {
    LooseAlong<E, TM> a(x, ks, ms, ks);
    if constexpr (kForm == kForward) {
      LooseAlong<E, TN> b(w + (int64_t)n0 * ks, ks, ns - n0, ks);
      tile_split<T, TM, TN>(a, b, nk, smem, false, store, store);
    } else {
      LooseAcross<E, TN> b(w + n0, ns, ns - n0, ks);
      tile_split<T, TM, TN>(a, b, nk, smem, false, store, store);
    }
  } else {
    Copied<SlabAlong<TM, TM / 8>> a(x, (int64_t)ks * sizeof(E), ms, 0, lane);
    if constexpr (kForm == kForward) {
      Copied<SlabAlong<TN, TN / 8>> b(w + (int64_t)n0 * ks, (int64_t)ks * sizeof(E), ns - n0, 0, lane);
      tile_split<T, TM, TN>(a, b, nk, smem, false, store, store);
    } else {
      Copied<SlabAcross<TN, TN / 8>> b(w + n0, (int64_t)ns * sizeof(E), ns - n0, ks, 0, lane);
      tile_split<T, TM, TN>(a, b, nk, smem, false, store, store);
    }
  }
}

template <class T, int kForm, int TM, int TN, bool kLoose>
__global__ __launch_bounds__(64 * kSplitWaves) void k_rows_split(ProductArgs p) {
  extern __shared__ __attribute__((aligned(16))) uint8_t smem[];
  const int ns = kForm == kForward ? p.O : p.I, tiles_n = (ns + TN - 1) / TN;
  PanelPlace at;
  if (!find_panel(p.rows, TM, blockIdx.x / (unsigned)tiles_n, at)) return;
  int tm, tn;
  tile_at(lin_of((int)(blockIdx.x - at.before * tiles_n), at.panels * tiles_n), at.panels, tiles_n, tm, tn);
  const int64_t first = at.first + (int64_t)tm * TM;
  const int ms = (int)min(at.end - first, (int64_t)TM);
  if (TM > 16 && ms <= 16)
    rows_split<T, kForm, 16, TN, kLoose>(p, at.group, first, ms, tn * TN, smem);
  else
    rows_split<T, kForm, TM, TN, kLoose>(p, at.group, first, ms, tn * TN, smem);
}

constexpr int kSumTile = 64;   // of the small tiles

// Four consecutive columns of row m of a group's sum, those in bounds.
__device__ __forceinline__ void store_sums(const ProductArgs& p, int e, int m, int n, f32x4 v) {
  if (m >= p.O || n >= p.I) return;
  const int64_t at = ((int64_t)e * p.O + m) * p.I + n;
  if (p.accumulate) {
    const float* sums = static_cast<const float*>(p.out) + at;
#pragma unroll
    for (int c = 0; c < 4; ++c) v[c] += n + c < p.I ? sums[c] : 0.f;
  }
  store_four(p.out, p.out_dtype, at, v, p.I - n, p.vector_out);
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
  tile_results<S>(acc, [&](int m, int n, f32x4 v) { store_sums(p, e, m0 + m, n0 + n, v); });
  if (!mirror) return;
  const int64_t out0 = (int64_t)e * p.O * p.I;
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

// The same as a small tile.
template <class T, bool kLoose>
__device__ __forceinline__ void sum_split(const ProductArgs& p, int e, int m0, int n0, bool mirror, uint8_t* smem) {
  using E = typename T::elem;
  constexpr int S = kSumTile;
  const int lane = threadIdx.x & 63;
  int64_t first, end;
  group_rows(p.rows, e, first, end);
  const int ks = (int)(end - first), nk = (ks + kSlabRows - 1) / kSlabRows;
  const E* dy = static_cast<const E*>(p.a) + first * p.O + m0;
  const E* x = static_cast<const E*>(p.b) + first * p.I + n0;
  const auto store = [&](int m, int n, f32x4 v) { store_sums(p, e, m0 + m, n0 + n, v); };
  const auto store_mirror = [&](int n, int m, f32x4 v) { store_sums(p, e, n0 + n, m0 + m, v); };
  if constexpr (kLoose) {
    LooseAcross<E, S> a(dy, p.O, p.O - m0, ks), b(x, p.I, p.I - n0, ks);
    tile_split<T, S, S>(a, b, nk, smem, mirror, store, store_mirror);
  } else {
    Copied<SlabAcross<S, S / 8>> a(dy, (int64_t)p.O * 2, p.O - m0, ks, 0, lane), b(x, (int64_t)p.I * 2, p.I - n0, ks, 0, lane);
    tile_split<T, S, S>(a, b, nk, smem, mirror, store, store_mirror);
  }
}

// A group's tiles of a sum, spread over the XCDs: all of dW; of H those on and above the diagonal (their
// transposes are stored too).  Of H's T tile rows, row r (T - r tiles) and row T - 1 - r (r + 1) are taken as
// one row of T + 1, so that the order of a rectangle serves; an odd T's middle row has the second half of its
// own empty.  False: none.
__device__ __forceinline__ bool find_sum_tile(const ProductArgs& p, int size, bool gram, int& e, int& m0, int& n0) {
  const int side = (p.I + size - 1) / size;
  const int tiles_m = gram ? (side + 1) / 2 : (p.O + size - 1) / size, tiles_n = gram ? side + 1 : side;
  const unsigned tiles = (unsigned)tiles_m * tiles_n;
  e = blockIdx.x / tiles;
  int tm, tn;
  tile_at(lin_of(blockIdx.x - e * tiles, tiles), tiles_m, tiles_n, tm, tn);
  if (gram) {
    const int r = tm, c = tn;
    tn = r + c;
    if (c >= side - r) {
      tm = side - 1 - r;
      tn = tm + c - (side - r);
      if (tm == r) return false;
    }
  }
  m0 = tm * size;
  n0 = tn * size;
  return true;
}

template <class T, bool kGram>
__global__ __launch_bounds__(256, 1) void k_sums_tile(ProductArgs p) {
  extern __shared__ __attribute__((aligned(16))) uint8_t smem[];
  int e, m0, n0;
  if (find_sum_tile(p, Whole::TM, kGram, e, m0, n0)) sum_tile<T>(p, e, m0, n0, kGram && m0 != n0, smem);
}

template <class T, bool kGram, bool kLoose>
__global__ __launch_bounds__(64 * kSplitWaves) void k_sums_split(ProductArgs p) {
  extern __shared__ __attribute__((aligned(16))) uint8_t smem[];
  int e, m0, n0;
  if (find_sum_tile(p, kSumTile, kGram, e, m0, n0)) sum_split<T, kLoose>(p, e, m0, n0, kGram && m0 != n0, smem);
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

int path() { static const char* h = getenv("GSQ_PATH"); return h ? atoi(h) : 0; }

template <class T, int kForm, int TM, int TN, bool kLoose>
hipError_t launch_rows_split(const ProductArgs& p, hipStream_t s) {
  const int ks = kForm == kForward ? p.I : p.O, ns = kForm == kForward ? p.O : p.I;
  const int nk = tiles_of(ks, ROW_BYTES / (int)sizeof(typename T::elem));
  const int waves = std::min(nk, kSplitWaves);
  return launch_lds<k_rows_split<T, kForm, TM, TN, kLoose>>(most_panels(p.rows, TM) * tiles_of(ns, TN), 64 * waves,
                    waves * (TM + TN) * ROW_BYTES, s, p);
}

template <class T, int kForm, bool kLoose>
hipError_t launch_rows_split(const ProductArgs& p, hipStream_t s) {
  const int ns = kForm == kForward ? p.O : p.I;
  const int64_t groups = std::min<int64_t>(p.rows.rows, p.rows.groups);
  const bool few = p.rows.rows <= 16 * groups, wide = most_panels(p.rows, few ? 16 : 64) * tiles_of(ns, 64) >= 256;
  if (few) return wide ? launch_rows_split<T, kForm, 16, 64, kLoose>(p, s) : launch_rows_split<T, kForm, 16, 16, kLoose>(p, s);
  return wide ? launch_rows_split<T, kForm, 64, 64, kLoose>(p, s) : launch_rows_split<T, kForm, 64, 16, kLoose>(p, s);
}

template <class T, int kForm>
hipError_t launch_rows(ProductArgs p, hipStream_t s) {
  if (p.rows.rows == 0) return hipSuccess;
  const int ns = kForm == kForward ? p.O : p.I;
  const int64_t unit = 16 / (int64_t)sizeof(typename T::elem);
  p.vector_out = four_at_once(p.out, p.out_dtype, ns);
  const bool tight = p.O % (kForm == kForward ? 1 : unit) == 0 && p.I % unit == 0 && aligned16(p.a) && aligned16(p.b);
  if (!tight) return launch_rows_split<T, kForm, true>(p, s);
  p.height = pick_height(p.rows, ns);
  const int64_t tiles = most_panels(p.rows, p.height) * tiles_of(ns, Whole::TN);
  if (path() == 2 || (path() == 0 && tiles < 128)) return launch_rows_split<T, kForm, false>(p, s);
  return launch_ring<k_rows_tile<T, kForm>>(tiles, s, p);
}

template <class T, bool kGram>
hipError_t launch_sums(ProductArgs p, hipStream_t s) {
  p.vector_out = four_at_once(p.out, p.out_dtype, p.I);
  const auto count = [&](int64_t tile) {
    const int64_t tm = tiles_of(p.O, tile), tn = tiles_of(p.I, tile);
    return p.rows.groups * (kGram ? (tn + 1) / 2 * (tn + 1) : tm * tn);
  };
  const bool tight = p.O % 8 == 0 && p.I % 8 == 0 && aligned16(p.a) && aligned16(p.b);
  if (tight && (path() == 1 || (path() == 0 && count(Whole::TM) >= 128 && p.rows.rows >= 128 * (int64_t)p.rows.groups)))
    return launch_ring<k_sums_tile<T, kGram>>(count(Whole::TM), s, p);
  const int waves = (int)std::max<int64_t>(1, std::min<int64_t>(kSplitWaves, (p.rows.rows + 63) / 64));
  const size_t lds = waves * 2 * kSumTile * ROW_BYTES;
  return tight ? launch_lds<k_sums_split<T, kGram, false>>(count(kSumTile), 64 * waves, lds, s, p)
               : launch_lds<k_sums_split<T, kGram, true>>(count(kSumTile), 64 * waves, lds, s, p);
}

}  // namespace

hipError_t launch_product(int form, int dtype, const ProductArgs& p, hipStream_t s) {
  const bool bf16 = dtype == GSQ_DT_BF16;
  if (form == kForward) return bf16 ? launch_rows<Bf16, kForward>(p, s) : launch_rows<F16, kForward>(p, s);
  if (form == kInputGrad) return bf16 ? launch_rows<Bf16, kInputGrad>(p, s) : launch_rows<F16, kInputGrad>(p, s);
  return bf16 ? launch_sums<Bf16, false>(p, s) : launch_sums<F16, false>(p, s);
}

hipError_t launch_product_i8(const ProductArgs& p, hipStream_t s) { return launch_rows<I8, kForward>(p, s); }

hipError_t launch_gram(int dtype, const ProductArgs& p, hipStream_t s) {
  return dtype == GSQ_DT_BF16 ? launch_sums<Bf16, true>(p, s) : launch_sums<F16, true>(p, s);
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
