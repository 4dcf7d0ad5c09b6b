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

// The values of both rows of a pair (16 lanes each), or of both halves, in every lane of them.
template <int kWidth>
__device__ __forceinline__ void both_rows(uint32_t v, uint32_t& a, uint32_t& b) {
  typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));
  u32x2 r;
  if constexpr (kWidth == 16)
    r = __builtin_amdgcn_permlane16_swap(v, v, false, false);
  else
    r = __builtin_amdgcn_permlane32_swap(v, v, false, false);
  a = r[0];
  b = r[1];
}
template <int kWidth>
__device__ __forceinline__ void both_rows(float v, float& a, float& b) {
  uint32_t x, y;
  both_rows<kWidth>(__float_as_uint(v), x, y);
  a = __uint_as_float(x);
  b = __uint_as_float(y);
}
template <int kWidth>
__device__ __forceinline__ void both_rows(double v, double& a, double& b) {
  const uint64_t u = __builtin_bit_cast(uint64_t, v);
  uint32_t x[2], y[2];
  both_rows<kWidth>((uint32_t)u, x[0], y[0]);
  both_rows<kWidth>((uint32_t)(u >> 32), x[1], y[1]);
  a = __builtin_bit_cast(double, (uint64_t)x[1] << 32 | x[0]);
  b = __builtin_bit_cast(double, (uint64_t)y[1] << 32 | y[0]);
}

// op over `LANES` neighbours: within a row by its own operations (lanes 1 and 2 apart, then mirrored in eight and in
// sixteen, when both sides of each mirror are alike), then over rows.
template <int LANES, class T, class Op>
__device__ __forceinline__ T over_lanes(T v, Op op) {
  static_assert(LANES == 16 || LANES == 64, "a row, or all lanes");
  v = op(v, of_lane<0xb1>(v));
  v = op(v, of_lane<0x4e>(v));
  v = op(v, of_lane<0x141>(v));
  v = op(v, of_lane<0x140>(v));
  if constexpr (LANES == 64) {
    T a, b;
    both_rows<16>(v, a, b);
    v = op(a, b);
    both_rows<32>(v, a, b);
    v = op(a, b);
  }
  return v;
}
template <int LANES, class T>
__device__ __forceinline__ T sum_lanes(T v) {
  return over_lanes<LANES>(v, [](T a, T b) { return a + b; });
}
// Maxima of values that are not NaN, by one instruction each (the compiler would quiet NaN first).
__device__ __forceinline__ float max_of(float a, float b) {
  float r;
  asm("v_max_f32 %0, %1, %2" : "=v"(r) : "v"(a), "v"(b));
  return r;
}
__device__ __forceinline__ double max_of(double a, double b) {
  double r;
  asm("v_max_f64 %0, %1, %2" : "=v"(r) : "v"(a), "v"(b));
  return r;
}
template <int LANES, class T>
__device__ __forceinline__ T max_lanes(T v) {
  return over_lanes<LANES>(v, [](T a, T b) { return max_of(a, b); });
}

}  // namespace
}  // namespace gsq
