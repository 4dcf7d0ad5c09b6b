// Device parts that the products of grouped rows share: element types and the search for a group's rows.
#pragma once
#include <hip/hip_runtime.h>
#include <stdint.h>

#include "gsq_plan.h"
#include "gsq_product.h"

namespace gsq {
namespace {

typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef int i32x4 __attribute__((ext_vector_type(4)));
typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef _Float16 f16x8 __attribute__((ext_vector_type(8)));

// Element types: what a matrix instruction of 16 x 16 outputs takes and sums into.
struct Bf16 {
  using elem = __bf16;
  using out = __bf16;
  using frag = bf16x8;
  using acc = f32x4;
  static constexpr int kDtype = GSQ_DT_BF16;
  static __device__ __forceinline__ acc mfma(frag a, frag b, acc c) {
    return __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, b, c, 0, 0, 0);
  }
};
struct F16 {
  using elem = _Float16;
  using out = _Float16;
  using frag = f16x8;
  using acc = f32x4;
  static constexpr int kDtype = GSQ_DT_FP16;
  static __device__ __forceinline__ acc mfma(frag a, frag b, acc c) {
    return __builtin_amdgcn_mfma_f32_16x16x32_f16(a, b, c, 0, 0, 0);
  }
};
template <class Out>      // of the scaled sums
struct I8 {
  using elem = int8_t;
  using out = Out;
  using frag = i32x4;
  using acc = i32x4;
  static constexpr int kDtype = -1;
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
  int panels;               // of the group
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
      at.first = of_src(a);
      at.end = of_src(b);
      return true;
    }
    before += all;
  }
  return false;
}

inline int64_t most_panels(const GroupRows& g, int64_t height) { return gsq::most_panels(g.rows, g.groups, height); }

}  // namespace
}  // namespace gsq
