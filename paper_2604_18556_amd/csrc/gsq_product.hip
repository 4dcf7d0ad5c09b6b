// Products of rows that are grouped by layer (the tokens of each routed expert): the layer's output, the
// gradients of its input and weights, the Gram matrix of its inputs, and the output in 8-bit integers.
#include <hip/hip_runtime.h>

#include <algorithm>

#include "gsq_split.hpp"

namespace gsq {
namespace {

// Columns n0 .. of y or dx for the ms rows from `first`.
template <class T>
__device__ __forceinline__ ResultColumns<typename T::out> row_columns(const ProductArgs& p, int group, int64_t first,
                                                                      int ms, int ns, int n0) {
  ResultColumns<typename T::out> r{static_cast<typename T::out*>(p.out) + first * ns + n0, ns, ms, ns - n0,
                                   p.vector_out != 0};
  if constexpr (T::kDtype < 0) {
    r.row_scales = p.a_scales + first;
    r.col_scales = p.b_scales + (int64_t)group * p.O + n0;
  }
  return r;
}

// One tile of y or dx.
template <class T, int kForm, class S, bool kLoose = false>
__device__ __forceinline__ void rows_tile(const ProductArgs& p, const RowsTile& at, uint8_t* smem) {
  const int64_t first = at.first;
  const int ms = at.ms, n0 = at.n0;
  using E = typename T::elem;
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int ks = kForm == kForward ? p.I : p.O, ns = kForm == kForward ? p.O : p.I;
  const int nk = (int)(((int64_t)ks * sizeof(E) + ROW_BYTES - 1) / ROW_BYTES);
  const E* w = static_cast<const E*>(p.b) + (int64_t)at.group * p.O * p.I;
  const E* x = static_cast<const E*>(p.a) + first * ks;
  typename T::acc acc[S::MI][S::NJ];
  if constexpr (kLoose) {
    RingLoose<LooseAlong<E, S::TM, S::TM / 32>> a(x, ks, ms, ks, wave);
    if constexpr (kForm == kForward) {
      RingLoose<LooseAlong<E, S::TN, S::TN / 32>> b(w + (int64_t)n0 * ks, ks, ns - n0, ks, wave);
      tile_ring<T, S>(a, b, nk, acc, smem);
    } else {
      RingLoose<LooseAcross<E, S::TN, S::TN / 32>> b(w + n0, ns, ns - n0, ks, wave);
      tile_ring<T, S>(a, b, nk, acc, smem);
    }
  } else {
    SlabAlong<S::TM> a(x, (int64_t)ks * sizeof(E), ms, wave, lane);
    if constexpr (kForm == kForward) {
      SlabAlong<S::TN> b(w + (int64_t)n0 * ks, (int64_t)ks * sizeof(E), ns - n0, wave, lane);
      tile_ring<T, S>(a, b, nk, acc, smem);
    } else {
      SlabAcross<S::TN> b(w + n0, (int64_t)ns * sizeof(E), ns - n0, ks, wave, lane);
      tile_ring<T, S>(a, b, nk, acc, smem);
    }
  }
  const auto out = row_columns<T>(p, at.group, first, ms, ns, n0);
  tile_results<S>(acc, smem, out, false, out);
}

// y or dx.
template <class T, int kForm>
__global__ __launch_bounds__(256, 1) void k_rows_tile(ProductArgs p) {
  extern __shared__ __attribute__((aligned(16))) uint8_t smem[];
  RowsTile at;
  if (!find_rows_tile(p.rows, p.height, Whole::TN, kForm == kForward ? p.O : p.I, at)) return;
  if (at.ms > Half::TM)
    rows_tile<T, kForm, Whole>(p, at, smem);
  else if (at.ms > Low::TM)
    rows_tile<T, kForm, Half>(p, at, smem);
  else
    rows_tile<T, kForm, Low>(p, at, smem);
}

// From any addresses, by way of registers: a quarter tile, two to a CU, so that one's waits are the other's work.
template <class T, int kForm>
__global__ __launch_bounds__(256, 2) void k_rows_loose(ProductArgs p) {
  extern __shared__ __attribute__((aligned(16))) uint8_t smem[];
  RowsTile at;
  if (find_rows_tile(p.rows, Quarter::TM, Quarter::TN, kForm == kForward ? p.O : p.I, at))
    rows_tile<T, kForm, Quarter, true>(p, at, smem);
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
  const auto out = row_columns<T>(p, group, first, ms, ns, n0);
  if constexpr (kLoose) {
    LooseAlong<E, TM> a(x, ks, ms, ks, 0);
    if constexpr (kForm == kForward) {
      LooseAlong<E, TN> b(w + (int64_t)n0 * ks, ks, ns - n0, ks, 0);
      tile_split<T, TM, TN>(a, b, nk, smem, out, false, out);
    } else {
      LooseAcross<E, TN> b(w + n0, ns, ns - n0, ks, 0);
      tile_split<T, TM, TN>(a, b, nk, smem, out, false, out);
    }
  } else {
    Copied<SlabAlong<TM, TM / 8>> a(x, (int64_t)ks * sizeof(E), ms, 0, lane);
    if constexpr (kForm == kForward) {
      Copied<SlabAlong<TN, TN / 8>> b(w + (int64_t)n0 * ks, (int64_t)ks * sizeof(E), ns - n0, 0, lane);
      tile_split<T, TM, TN>(a, b, nk, smem, out, false, out);
    } else {
      Copied<SlabAcross<TN, TN / 8>> b(w + n0, (int64_t)ns * sizeof(E), ns - n0, ks, 0, lane);
      tile_split<T, TM, TN>(a, b, nk, smem, out, false, out);
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

// Columns n0 .. of a group's sum for the rows from m0.
template <class Out>
__device__ __forceinline__ ResultColumns<Out> sum_columns(const ProductArgs& p, int e, int m0, int n0) {
  return {static_cast<Out*>(p.out) + ((int64_t)e * p.O + m0) * p.I + n0, p.I, p.O - m0, p.I - n0, p.vector_out != 0,
          p.accumulate != 0};
}

// One tile of a sum over a group's rows: out[m0 .., n0 ..] (+)= sum_r a[r, m] b[r, n], and with `mirror` its
// transpose too.
template <class T, class Out, class S, bool kLoose>
__device__ __forceinline__ void sum_tile(const ProductArgs& p, int e, int m0, int n0, bool mirror, uint8_t* smem) {
  using E = typename T::elem;
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  int64_t first, end;
  group_rows(p.rows, e, first, end);
  const int ks = (int)(end - first), nk = (ks + kSlabRows - 1) / kSlabRows;
  const E* dy = static_cast<const E*>(p.a) + first * p.O + m0;   // without rows, only zeros are read
  const E* x = static_cast<const E*>(p.b) + first * p.I + n0;
  typename T::acc acc[S::MI][S::NJ];
  if constexpr (kLoose) {
    RingLoose<LooseAcross<E, S::TM, S::TM / 32>> a(dy, p.O, p.O - m0, ks, wave), b(x, p.I, p.I - n0, ks, wave);
    tile_ring<T, S>(a, b, nk, acc, smem);
  } else {
    SlabAcross<S::TM> a(dy, (int64_t)p.O * 2, p.O - m0, ks, wave, lane), b(x, (int64_t)p.I * 2, p.I - n0, ks, wave, lane);
    tile_ring<T, S>(a, b, nk, acc, smem);
  }
  tile_results<S>(acc, smem, sum_columns<Out>(p, e, m0, n0), mirror, sum_columns<Out>(p, e, n0, m0));
}

// The same as a small tile.
template <class T, class Out, int S, bool kLoose>
__device__ __forceinline__ void sum_split(const ProductArgs& p, int e, int m0, int n0, bool mirror, uint8_t* smem) {
  using E = typename T::elem;
  const int lane = threadIdx.x & 63;
  int64_t first, end;
  group_rows(p.rows, e, first, end);
  const int ks = (int)(end - first), nk = (ks + kSlabRows - 1) / kSlabRows;
  const E* dy = static_cast<const E*>(p.a) + first * p.O + m0;
  const E* x = static_cast<const E*>(p.b) + first * p.I + n0;
  const auto out = sum_columns<Out>(p, e, m0, n0), turned = sum_columns<Out>(p, e, n0, m0);
  if constexpr (kLoose) {
    LooseAcross<E, S> a(dy, p.O, p.O - m0, ks, 0), b(x, p.I, p.I - n0, ks, 0);
    tile_split<T, S, S>(a, b, nk, smem, out, mirror, turned);
  } else {
    Copied<SlabAcross<S, S / 8>> a(dy, (int64_t)p.O * 2, p.O - m0, ks, 0, lane), b(x, (int64_t)p.I * 2, p.I - n0, ks, 0, lane);
    tile_split<T, S, S>(a, b, nk, smem, out, mirror, turned);
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

template <class T, class Out, bool kGram, class S, bool kLoose>
__global__ __launch_bounds__(256, S::LDS > LDS_BYTES / 2 ? 1 : 2) void k_sums_tile(ProductArgs p) {
  extern __shared__ __attribute__((aligned(16))) uint8_t smem[];
  int e, m0, n0;
  if (find_sum_tile(p, S::TM, kGram, e, m0, n0)) sum_tile<T, Out, S, kLoose>(p, e, m0, n0, kGram && m0 != n0, smem);
}

template <class T, class Out, bool kGram, int S, bool kLoose>
__global__ __launch_bounds__(64 * kSplitWaves) void k_sums_split(ProductArgs p) {
  extern __shared__ __attribute__((aligned(16))) uint8_t smem[];
  int e, m0, n0;
  if (find_sum_tile(p, S, kGram, e, m0, n0)) sum_split<T, Out, S, kLoose>(p, e, m0, n0, kGram && m0 != n0, smem);
}

// Rows in 8-bit integers: s = max |x| / 127 in fp32, q = x / s to the nearest integer, ties to even.  A
// row of zeros has s = 0 and q = 0; a row with an infinity or NaN s = NaN and q = 0, so that its products
// are NaN.  A row is read once: up to kHeld chunks of 16 values stay with each thread, what is longer is read
// again.  Chunks begin at multiples of 16 values; from any address, by unaligned loads and stores.
constexpr int kHeld = 2, kChunk = 16;

template <class E>
struct QuantChunk {
  E v[kChunk];
  __device__ __forceinline__ void load(const E* x, int64_t c, int64_t cols) {
    if (c + kChunk <= cols) {
      __builtin_memcpy(v, x + c, sizeof(v));
    } else {
#pragma unroll
      for (int i = 0; i < kChunk; ++i) v[i] = c + i < cols ? x[c + i] : (E)0;
    }
  }
  // The largest magnitude as its bits, which order like the values; infinities and NaN lie above all others.
  __device__ __forceinline__ uint32_t top() const {
    uint32_t t = 0;
#pragma unroll
    for (int i = 0; i < kChunk; ++i) t = max(t, __float_as_uint((float)v[i]) & 0x7fffffffu);
    return t;
  }
  // x, s and 1 / s, with x and s scaled by `by`.
  __device__ __forceinline__ void write(int8_t* q, int64_t c, int64_t cols, float s, float inv, float by) const {
    int8_t out[kChunk];
#pragma unroll
    for (int i = 0; i < kChunk; ++i) {
      const float x = inv == 0.f ? 0.f : (float)v[i] * by;
      // x times a reciprocal may round onto a half, off it, or past it: the remainder, exact in an fma, decides
      float r = rintf(x * inv);
      const float rest = fmaf(-r, s, x), twice = 2.f * fabsf(rest);
      if (twice > s || (twice == s && ((int)r & 1))) r += copysignf(1.f, rest);
      out[i] = (int8_t)(int)fminf(fmaxf(r, -127.f), 127.f);
    }
    if (c + kChunk <= cols) {
      __builtin_memcpy(q + c, out, sizeof(out));
    } else {
#pragma unroll
      for (int i = 0; i < kChunk; ++i)
        if (c + i < cols) q[c + i] = out[i];
    }
  }
};

template <class E>
__global__ __launch_bounds__(256) void k_quantize_rows(const E* __restrict__ x, int64_t cols,
                                                       int8_t* __restrict__ q, float* __restrict__ scales) {
  __shared__ uint32_t part[4];
  const int64_t row = blockIdx.x;
  x += row * cols;
  q += row * cols;
  const int64_t c0 = (int64_t)threadIdx.x * kChunk, step = (int64_t)blockDim.x * kChunk;
  QuantChunk<E> held[kHeld];
  uint32_t top = 0;
#pragma unroll
  for (int h = 0; h < kHeld; ++h) {
    held[h].load(x, min(c0 + h * step, cols), cols);
    top = max(top, held[h].top());
  }
  for (int64_t c = c0 + kHeld * step; c < cols; c += step) {
    QuantChunk<E> more;
    more.load(x, c, cols);
    top = max(top, more.top());
  }
#pragma unroll
  for (int d = 32; d; d >>= 1) top = max(top, (uint32_t)__shfl_xor((int)top, d, 64));
  if (blockDim.x > 64) {
    if ((threadIdx.x & 63) == 0) part[threadIdx.x >> 6] = top;
    __syncthreads();
    for (unsigned w = 0; w < blockDim.x >> 6; ++w) top = max(top, part[w]);
  }
  const float s = top >= 0x7f800000u ? __builtin_nanf("") : __uint_as_float(top) / 127.f;
  if (threadIdx.x == 0) scales[row] = s;
  const bool some = s > 0.f;   // else every q is zero: nothing is divided by zero or NaN
  // the reciprocal of a very small scale would overflow: row and scale are taken 2^24 times as large
  const float tiny = s < 1e-37f ? 0x1p24f : 1.f;
  const float sc = some ? s * tiny : 1.f, inv = some ? 1.f / sc : 0.f;
#pragma unroll
  for (int h = 0; h < kHeld; ++h)
    if (c0 + h * step < cols) held[h].write(q, c0 + h * step, cols, sc, inv, tiny);
  for (int64_t c = c0 + kHeld * step; c < cols; c += step) {
    QuantChunk<E> more;
    more.load(x, c, cols);
    more.write(q, c, cols, sc, inv, tiny);
  }
}

template <class T, int kForm, int TM, int TN, bool kLoose>
hipError_t launch_rows_split(const ProductArgs& p, hipStream_t s) {
  const int ks = kForm == kForward ? p.I : p.O, ns = kForm == kForward ? p.O : p.I;
  const int nk = (int)tiles_of(ks, ROW_BYTES / (int)sizeof(typename T::elem));
  const int waves = std::min(nk, kSplitWaves);
  return launch_lds<k_rows_split<T, kForm, TM, TN, kLoose>>(most_panels(p.rows, TM) * tiles_of(ns, TN), 64 * waves,
                    waves * (TM + TN) * ROW_BYTES, s, p);
}

template <class T, int kForm, bool kLoose>
hipError_t launch_rows_split(const ProductArgs& p, const RowsPlan& plan, hipStream_t s) {
  if (plan.height == 16)
    return plan.width == 64 ? launch_rows_split<T, kForm, 16, 64, kLoose>(p, s)
                            : launch_rows_split<T, kForm, 16, 16, kLoose>(p, s);
  return plan.width == 64 ? launch_rows_split<T, kForm, 64, 64, kLoose>(p, s)
                          : launch_rows_split<T, kForm, 64, 16, kLoose>(p, s);
}

template <class T, int kForm>
hipError_t launch_rows(ProductArgs p, hipStream_t s) {
  if (p.rows.rows == 0) return hipSuccess;
  const int ns = kForm == kForward ? p.O : p.I, ks = kForm == kForward ? p.I : p.O;
  const int64_t unit = 16 / (int64_t)sizeof(typename T::elem);
  const int slabs = (int)tiles_of(ks, ROW_BYTES / (int)sizeof(typename T::elem));
  p.vector_out = four_at_once(p.out, p.out_dtype, ns);
  const bool tight = p.O % (kForm == kForward ? 1 : unit) == 0 && p.I % unit == 0 && aligned16(p.a) && aligned16(p.b);
  const RowsPlan plan = plan_rows(p.rows.rows, p.rows.groups, ns, slabs, tight, kForm == kInputGrad, T::kDtype < 0);
  if (!plan.height) return hipErrorInvalidConfiguration;
  if (plan.split) return tight ? launch_rows_split<T, kForm, false>(p, plan, s) : launch_rows_split<T, kForm, true>(p, plan, s);
  if (!tight)
    return launch_lds<k_rows_loose<T, kForm>>(most_panels(p.rows, Quarter::TM) * tiles_of(ns, Quarter::TN), 256,
                                              Quarter::LDS, s, p);
  p.height = plan.height;
  return launch_ring<k_rows_tile<T, kForm>>(most_panels(p.rows, p.height) * tiles_of(ns, Whole::TN), s, p);
}

template <class T, class Out, bool kGram>
hipError_t launch_sums(ProductArgs p, hipStream_t s) {
  p.vector_out = four_at_once(p.out, p.out_dtype, p.I);
  const bool tight = p.O % 8 == 0 && p.I % 8 == 0 && aligned16(p.a) && aligned16(p.b);
  const SumsPlan plan = plan_sums(p.rows.rows, p.rows.groups, p.O, p.I, tight, kGram);
  const int64_t tiles = sum_tiles(p.rows.groups, p.O, p.I, kGram, plan.size);
  if (!plan.split && plan.size == Whole::TM)
    return launch_lds<k_sums_tile<T, Out, kGram, Whole, false>>(tiles, 256, Whole::LDS, s, p);
  if (!plan.split)
    return tight ? launch_lds<k_sums_tile<T, Out, kGram, Quarter, false>>(tiles, 256, Quarter::LDS, s, p)
                 : launch_lds<k_sums_tile<T, Out, kGram, Quarter, true>>(tiles, 256, Quarter::LDS, s, p);
  const int waves = plan.waves;
  const auto launch = [&](auto size, auto loose) {
    constexpr int S = decltype(size)::value;
    return launch_lds<k_sums_split<T, Out, kGram, S, decltype(loose)::value>>(tiles, 64 * waves, (size_t)waves * 2 * S * ROW_BYTES,
                                                                         s, p);
  };
  using Is64 = std::integral_constant<int, 64>;
  using Is32 = std::integral_constant<int, 32>;
  if (plan.size == 32) return tight ? launch(Is32{}, std::false_type{}) : launch(Is32{}, std::true_type{});
  return tight ? launch(Is64{}, std::false_type{}) : launch(Is64{}, std::true_type{});
}

}  // namespace

hipError_t launch_product(int form, int dtype, const ProductArgs& p, hipStream_t s) {
  const bool bf16 = dtype == GSQ_DT_BF16;
  if (form == kForward) return bf16 ? launch_rows<Bf16, kForward>(p, s) : launch_rows<F16, kForward>(p, s);
  if (form == kInputGrad) return bf16 ? launch_rows<Bf16, kInputGrad>(p, s) : launch_rows<F16, kInputGrad>(p, s);
  if (p.out_dtype == GSQ_DT_FP32)
    return bf16 ? launch_sums<Bf16, float, false>(p, s) : launch_sums<F16, float, false>(p, s);
  return bf16 ? launch_sums<Bf16, __bf16, false>(p, s) : launch_sums<F16, _Float16, false>(p, s);
}

hipError_t launch_product_i8(const ProductArgs& p, hipStream_t s) {
  return p.out_dtype == GSQ_DT_BF16 ? launch_rows<I8<__bf16>, kForward>(p, s) : launch_rows<I8<_Float16>, kForward>(p, s);
}

hipError_t launch_gram(int dtype, const ProductArgs& p, hipStream_t s) {
  return dtype == GSQ_DT_BF16 ? launch_sums<Bf16, float, true>(p, s) : launch_sums<F16, float, true>(p, s);
}

hipError_t launch_quantize_rows(const void* x, int dtype, int64_t rows, int64_t cols, int8_t* q,
                                float* scales, hipStream_t s) {
  if (rows == 0) return hipSuccess;
  const int threads = (int)std::min<int64_t>(256, (cols + 64 * kChunk - 1) / (64 * kChunk) * 64);
  if (dtype == GSQ_DT_BF16)
    k_quantize_rows<<<rows, threads, 0, s>>>(static_cast<const __bf16*>(x), cols, q, scales);
  else if (dtype == GSQ_DT_FP16)
    k_quantize_rows<<<rows, threads, 0, s>>>(static_cast<const _Float16*>(x), cols, q, scales);
  else
    k_quantize_rows<<<rows, threads, 0, s>>>(static_cast<const float*>(x), cols, q, scales);
  return hipGetLastError();
}

}  // namespace gsq
