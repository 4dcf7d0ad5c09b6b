// How wavefronts share the slabs of rows that come in several segments.  Plain C++, apart from the kernel that walks so,
// that it can be tested without a GPU.
#pragma once
#include <stdint.h>

namespace gsq {

// One wavefront's walk: of the slabs of all segments together, counted anew in each, it takes number `skip` and then
// every `every`-th.
struct SlabWalk {
  int64_t skip;                // slabs to its next one
  int64_t at = 0, end = 0;     // rows of the present segment that are left
  constexpr explicit SlabWalk(int64_t before) : skip(before) {}
  constexpr void enter(int64_t first, int64_t last) {
    at = first;
    end = last;
  }
  // Its next slab of the present segment: the first row, and how many it has.  Where there is none the segment is done:
  // asked again, there is none either.
  constexpr bool take(int height, int every, int64_t& first, int& rows) {
    const int64_t left = (end - at + height - 1) / height;
    if (skip >= left) {
      skip -= left;
      at = end;
      return false;
    }
    at += skip * height;
    first = at;
    rows = end - at < height ? (int)(end - at) : height;
    skip = every;
    return true;
  }
};

}  // namespace gsq
