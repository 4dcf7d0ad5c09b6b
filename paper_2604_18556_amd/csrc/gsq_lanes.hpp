// Sums and maxima over groups of 16 or 64 neighbouring lanes, each lane having the result.
#pragma once
#include <hip/hip_runtime.h>
#include <stdint.h>

namespace gsq {
namespace {

// The value of the lane that a row operation pairs with this one (rows have 16 lanes).
template <int kCtrl>
__device__ __forceinline__ uint32_t of_lane(uint32_t v) {
  return (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, kCtrl, 0xf, 0xf, true);
}
template <int kCtrl>
__device__ __forceinline__ float of_lane(float v) {
  return __uint_as_float(of_lane<kCtrl>(__float_as_uint(v)));
}
template <int kCtrl>
__device__ __forceinline__ double of_lane(double v) {
  const uint64_t b = __builtin_bit_cast(uint64_t, v);
  return __builtin_bit_cast(double, (uint64_t)of_lane<kCtrl>((uint32_t)(b >> 32)) << 32 | of_lane<kCtrl>((uint32_t)b));
}

// op over `LANES` neighbours: within a row by its own operations (lanes 1 and 2 apart, then mirrored in eight and in
// sixteen, when both sides of each mirror are alike), across rows by way of LDS.
template <int LANES, class T, class Op>
__device__ __forceinline__ T over_lanes(T v, Op op) {
  static_assert(LANES == 16 || LANES == 64, "a row, or all lanes");
  v = op(v, of_lane<0xb1>(v));
  v = op(v, of_lane<0x4e>(v));
  v = op(v, of_lane<0x141>(v));
  v = op(v, of_lane<0x140>(v));
  if constexpr (LANES == 64) {
    v = op(v, __shfl_xor(v, 16, 64));
    v = op(v, __shfl_xor(v, 32, 64));
  }
  return v;
}
template <int LANES, class T>
__device__ __forceinline__ T sum_lanes(T v) {
  return over_lanes<LANES>(v, [](T a, T b) { return a + b; });
}
template <int LANES, class T>
__device__ __forceinline__ T max_lanes(T v) {
  return over_lanes<LANES>(v, [](T a, T b) { return a > b ? a : b; });
}

}  // namespace
}  // namespace gsq
