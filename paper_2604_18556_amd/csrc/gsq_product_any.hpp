// Device parts that the products of grouped rows share: element types, the search for a group's rows,
// and the product of one 64 x 64 tile from any operands.
#pragma once
#include <hip/hip_runtime.h>
#include <stdint.h>

#include "gsq_product.h"

namespace gsq {
namespace {

typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef int i32x4 __attribute__((ext_vector_type(4)));
typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef _Float16 f16x8 __attribute__((ext_vector_type(8)));

// Element types: what a matrix instruction of 16 x 16 x kStep takes and sums into.
struct Bf16 {
  using elem = __bf16;
  using frag = bf16x8;
  using acc = f32x4;
  static constexpr int kStep = 32, kDtype = GSQ_DT_BF16;
  static __device__ __forceinline__ acc mfma(frag a, frag b, acc c) {
    return __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, b, c, 0, 0, 0);
  }
};
struct F16 {
  using elem = _Float16;
  using frag = f16x8;
  using acc = f32x4;
  static constexpr int kStep = 32, kDtype = GSQ_DT_FP16;
  static __device__ __forceinline__ acc mfma(frag a, frag b, acc c) {
    return __builtin_amdgcn_mfma_f32_16x16x32_f16(a, b, c, 0, 0, 0);
  }
};
struct I8 {
  using elem = int8_t;
  using frag = i32x4;
  using acc = i32x4;
  static constexpr int kStep = 64, kDtype = -1;
  static __device__ __forceinline__ acc mfma(frag a, frag b, acc c) {
    return __builtin_amdgcn_mfma_i32_16x16x64_i8(a, b, c, 0, 0, 0);
  }
};

// Rows of group e.  Offsets outside [0, rows] or falling ones are read as the nearest that are not, so
// that nothing outside the arrays is touched whatever the device memory holds.
__device__ __forceinline__ void group_rows(const GroupRows& g, int e, int64_t& first, int64_t& end) {
  first = 0;
  end = g.rows;
  if (g.offsets) {
    first = min(max(g.offsets[e], (int64_t)0), g.rows);
    end = min(max(g.offsets[e + 1], first), g.rows);
  }
}

// Where a workgroup stands when every group's rows are cut into panels of equal height, group after group.
struct PanelPlace {
  int group;
  int panel, panels;        // in the group
  int64_t first, end;       // rows of the group
  int64_t before;           // panels of the groups before it
};

// Panel `index` of all groups.  False: there are fewer.  The whole wavefront calls it; 64 groups are counted
// at a time.  Taking all full panels before the groups' shorter rests instead (64 experts of 2048 x 7168,
// 16384 rows: 681 us against 640) parts the panels that are bound by the matrix cores from those that are bound
// by their weights' bytes, and reads many weights twice.
__device__ __forceinline__ bool find_panel(const GroupRows& g, int height, int64_t index, PanelPlace& at) {
  const int lane = threadIdx.x & 63;
  int64_t before = 0;
  for (int e0 = 0; e0 < g.groups; e0 += 64) {
    int64_t a = 0, b = 0;
    if (e0 + lane < g.groups) group_rows(g, e0 + lane, a, b);
    const int mine = (int)((b - a + height - 1) / height);
    int upto = mine;
#pragma unroll
    for (int d = 1; d < 64; d <<= 1) {
      const int x = __shfl_up(upto, d, 64);
      if (lane >= d) upto += x;
    }
    const int all = __builtin_amdgcn_readlane(upto, 63);
    if (index - before < all) {
      const int src = __builtin_ctzll(__ballot((int)(index - before) < upto));
      const auto of_src = [&](int64_t v) {
        const uint32_t lo = __builtin_amdgcn_readlane((uint32_t)v, src);
        const uint32_t hi = __builtin_amdgcn_readlane((uint32_t)(v >> 32), src);
        return (int64_t)((uint64_t)hi << 32 | lo);
      };
      at.group = e0 + src;
      at.panels = (int)of_src(mine);
      at.before = before + of_src(upto - mine);
      at.panel = (int)(index - at.before);
      at.first = of_src(a);
      at.end = of_src(b);
      return true;
    }
    before += all;
  }
  return false;
}

// Most panels there can be, for the grid.
inline int64_t most_panels(const GroupRows& g, int64_t height) {
  return g.rows / height + (g.rows < g.groups ? g.rows : g.groups);
}

// Output element: rounded once, to the nearest (ties to even).
__device__ __forceinline__ void store_out(void* out, int dtype, int64_t at, float v) {
  if (dtype == GSQ_DT_BF16)
    static_cast<__bf16*>(out)[at] = (__bf16)v;
  else if (dtype == GSQ_DT_FP16)
    static_cast<_Float16*>(out)[at] = (_Float16)v;
  else
    static_cast<float*>(out)[at] = v;
}

// Operands of the tile product, element by element: m is the output's row or column, k is summed over.
// Out of range they are zero.
template <class E>
struct AlongK {            // k is contiguous
  const E* p;
  int64_t ld;
  int ms, ks;
  static constexpr bool kFast = true;
  __device__ __forceinline__ E at(int m, int k) const { return m < ms && k < ks ? p[m * ld + k] : (E)0; }
};
template <class E>
struct AcrossK {           // m is contiguous
  const E* p;
  int64_t ld;
  int ms, ks;
  static constexpr bool kFast = false;
  __device__ __forceinline__ E at(int m, int k) const { return m < ms && k < ks ? p[k * ld + m] : (E)0; }
};

constexpr int kAnyTile = 64;

// One 64 x 64 tile at (m0, n0) of a product over ks, for operands of any size and alignment: elements
// go through registers into LDS, both operands as rows along k, 64 of k at a time, and the next slab is
// fetched while this one is multiplied.  Four wavefronts, 32 x 32 each.
// store(m, n, sum) is called for every element of the tile, also beyond the operands' sizes.
template <class T, class A, class B, class Store>
__device__ __forceinline__ void tile_any(const A& a, const B& b, int m0, int n0, int ks, Store store) {
  using E = typename T::elem;
  constexpr int BK = 64, ROW = BK + 16 / (int)sizeof(E);
  constexpr int PER = kAnyTile * BK / 256;
  __shared__ __align__(16) E As[kAnyTile * ROW], Bs[kAnyTile * ROW];
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  const int wm = (wave >> 1) * 32, wn = (wave & 1) * 32;

  typename T::acc acc[2][2] = {};
  E ra[PER], rb[PER];
  const auto fetch = [&](int k0) {
#pragma unroll
    for (int i = 0; i < PER; ++i) {
      const int f = i * 256 + tid, slow = f / 64, fast = f % 64;
      ra[i] = A::kFast ? a.at(m0 + slow, k0 + fast) : a.at(m0 + fast, k0 + slow);
      rb[i] = B::kFast ? b.at(n0 + slow, k0 + fast) : b.at(n0 + fast, k0 + slow);
    }
  };
  fetch(0);
  for (int k0 = 0; k0 < ks; k0 += BK) {
    __syncthreads();
#pragma unroll
    for (int i = 0; i < PER; ++i) {
      const int f = i * 256 + tid, slow = f / 64, fast = f % 64;
      As[A::kFast ? slow * ROW + fast : fast * ROW + slow] = ra[i];
      Bs[B::kFast ? slow * ROW + fast : fast * ROW + slow] = rb[i];
    }
    __syncthreads();
    if (k0 + BK < ks) fetch(k0 + BK);
#pragma unroll
    for (int h = 0; h < BK / T::kStep; ++h) {
      typename T::frag fa[2], fb[2];
#pragma unroll
      for (int i = 0; i < 2; ++i) {
        const int k = h * T::kStep + (lane >> 4) * (T::kStep / 4);
        fa[i] = *reinterpret_cast<const typename T::frag*>(&As[(wm + 16 * i + (lane & 15)) * ROW + k]);
        fb[i] = *reinterpret_cast<const typename T::frag*>(&Bs[(wn + 16 * i + (lane & 15)) * ROW + k]);
      }
#pragma unroll
      for (int i = 0; i < 2; ++i)
#pragma unroll
        for (int j = 0; j < 2; ++j) acc[i][j] = T::mfma(fa[i], fb[j], acc[i][j]);
    }
  }
  // lane l of a 16 x 16 block: column l % 16, rows 4 (l / 16) .. + 3
#pragma unroll
  for (int i = 0; i < 2; ++i)
#pragma unroll
    for (int j = 0; j < 2; ++j)
#pragma unroll
      for (int r = 0; r < 4; ++r)
        store(m0 + wm + 16 * i + 4 * (lane >> 4) + r, n0 + wn + 16 * j + (lane & 15), acc[i][j][r]);
}

}  // namespace
}  // namespace gsq
