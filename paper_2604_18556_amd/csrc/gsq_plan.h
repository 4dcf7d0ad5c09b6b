// Which tiles a product is cut into: rules on sizes, types and alignment.  Plain C++, apart from the kernels, so
// that what they choose can be read and tested without a GPU.
#pragma once
#include <stdint.h>

#include <algorithm>
#include <cmath>

namespace gsq {

inline int64_t tiles_of(int64_t n, int64_t tile) { return (n + tile - 1) / tile; }

// Most panels of `height` rows that the rows of all groups can make, for the grid.
inline int64_t most_panels(int64_t rows, int64_t groups, int64_t height) {
  return rows / height + std::min(rows, groups);
}

// What one launch holds: fewer than 2^32 threads in the grid's one dimension.
inline bool fits_launch(int64_t tiles, int64_t threads) { return tiles * threads < (int64_t)1 << 32; }

// Bytes of a packed layer as it is kept, in units of 16 channels x 128 inputs (64 lanes with 32 codes each); `gs`:
// inputs per fp16 scale, `super`: with sub-scales, a byte for each 16 inputs.
struct KeptBytes {
  int64_t codes, scales, sub;
};
inline KeptBytes kept_bytes(int64_t batch, int O, int I, int bits, int gs, bool super) {
  const int64_t tiles = batch * tiles_of(O, 16), blocks = tiles_of(I, 128), lanes = tiles * blocks * 64;
  return {lanes * bits * 4, gs == 16 ? lanes * 4 : tiles * tiles_of(blocks * 128, gs) * 32, super ? lanes * 2 : 0};
}

// Workgroups of 256 threads that lay out `count` elements of a packed layer.  From eight full GPUs' (256 CUs x 8) on
// they pass over the rest, so that a layer of any size fits a launch.  (64 super-block experts of 2048 x 7168: 1.85 ms,
// with a workgroup for every 256 elements 1.84, with one full GPU's 2.02.)
inline unsigned unpack_blocks(int64_t count) { return (unsigned)std::min<int64_t>(tiles_of(count, 256), 16384); }

// Wavefronts that share a tile's sum, at most: one for each of its slabs (packed codes: units) up to these.  Whole
// workgroups have four.
constexpr int kSplitWaves = 8, kFewWaves = 16, kRingWaves = 4;

// How a product of rows is cut: panels of `height` rows and `width` columns, by whole workgroups (ring) or by
// wavefronts that share the sum (split).  No height: nothing fits a launch.
struct RowsPlan {
  bool split;
  int height, width;
};

// Microseconds of a tile: its start, and each slab (128 bytes of k) on an empty GPU and with a tile on each of
// 256 CUs.
struct TileCost {
  int height, width;
  double start, alone, full;
};

// The cheapest of several tiles of `waves` wavefronts that fit one launch: a launch, and a tile's time for each round
// of 256 tiles.  The groups' last panels are taken to be half full, and `fewest` are reckoned with at least.
template <int N>
RowsPlan cheapest(int64_t rows, int64_t groups, int cols, int slabs, const TileCost (&costs)[N], bool split, int waves,
                  double& best, RowsPlan plan, double fewest = 0) {
  const double few = (double)std::min(rows, groups);
  for (const TileCost& c : costs) {
    if (!fits_launch(most_panels(rows, groups, c.height) * tiles_of(cols, c.width), 64 * waves)) continue;
    const double panels = groups == 1 ? (double)tiles_of(rows, c.height) : rows / (double)c.height + few / 2;
    const double tiles = std::max(panels, fewest) * tiles_of(cols, c.width), rounds = tiles / 256;
    const double whole = rounds < 1 ? 1 : groups == 1 ? (double)(int64_t)(rounds + 0.999) : rounds;
    const double each = c.alone + (c.full - c.alone) * (rounds < 1 ? rounds : 1);
    const double us = 4 + whole * (c.start + slabs * each);
    if (us < best) {
      best = us;
      plan = {split, c.height, c.width};
    }
  }
  return plan;
}

// y (or dx: across): whole workgroups on panels of 256, 128 or 64 rows, or wavefronts that share a sum.  `tight`: the
// operands' rows are aligned to 16 bytes; `bytes`: 8-bit integers.  The costs are fitted to bf16 products of one
// group (us for x W^T; 256 | 128 | 64 rows by workgroups, 64 x 64 | 64 x 16 split):
//   8192 x 8192: 64 rows - | - | 101, 44 | 51; 256 rows 154 | 111 | 100, 71 | 141; 512 rows 158 | 112 | 101,
//     125 | 246; 1024 rows 162 | 123 | 205, 225 | -; 2048 rows 208 | 242 | 371, 432 | -
//   2048 x 2048: 64 rows - | - | 18.1, 9.6 | 6.7; 512 rows 47 | 30 | 19, 11 | 19; 2048 rows 49 | 31 | 24, 38 | -
//   O 512, I 8192: 512 rows 147 | 90 | 57, 25 | 18; 4096 rows 150 | 92 | 60, 54 | -
// and 8192 x 8192 at one row by 16 x 64 | 16 x 16 split 30 | 28, at 64 rows 50 | 68.  8-bit integers take
// longer in large tiles, which the power of the matrix cores bounds.
inline RowsPlan plan_rows(int64_t rows, int64_t groups, int cols, int slabs, bool tight, bool across, bool bytes) {
  const int waves = std::min(slabs, kSplitWaves);
  double best = 1e30;
  if (!tight) {
    // from any addresses (I 4001, O 8190; 64 x 64 split | 128 x 128): 64 rows 32 | 72, 512 rows 118 | 78, 4096 rows
    // 866 | 378
    const TileCost small[] = {{64, 64, 1, 0.17, 0.42}, {64, 16, 1, 0.1, 0.21}, {16, 64, 1, 0.07, 0.15}, {16, 16, 0.5, 0.025, 0.08}};
    const TileCost large[] = {{128, 128, 2, across ? 2.0 : 0.85, across ? 1.05 : 0.75}};
    const RowsPlan plan = cheapest(rows, groups, cols, slabs, small, true, waves, best, RowsPlan{});
    return cheapest(rows, groups, cols, slabs, large, false, kRingWaves, best, plan);
  }
  const double more = bytes ? 1.4 : 1;
  const TileCost small[] = {{64, 64, 1, 0.165, 0.22}, {64, 16, 1, 0.1, 0.115}, {16, 64, 1, 0.06, 0.1}, {16, 16, 0.5, 0.02, 0.055}};
  const TileCost large[] = {{256, 256, 3, 1.15 * more, 1.6 * more}, {128, 256, 2, 0.7 * more, 0.95 * more},
                            {64, 256, 1.5, 0.43 * more, 0.72 * more}};
  const RowsPlan plan = cheapest(rows, groups, cols, slabs, small, true, waves, best, RowsPlan{});
  return cheapest(rows, groups, cols, slabs, large, false, kRingWaves, best, plan);
}

// y with the packed codes, by the same reckoning (us at 2 bits; 16 | 64 channels shared | panels of 64 | 128 | 256
// rows by workgroups):
//   I 4096, O 4096: 1 row 6 | 10 | 52 | - | -; 17 rows - | 10; 256 rows - | 17 | 55 | 72 | 96; 2048 rows - | 116 |
//     135 | 86 | 107; 4096 rows - | 219 | 247 | 152 | 113
//   I 4096, O 14336: 1 row - | 9 | 52; 64 rows - | 15 | 54; 512 rows - | 98 | 129 | 80 | 102; 1024 rows - | 188 |
//     246 | 150 | 107
//   I 14336, O 4096: 1 row 11 | 25 | 173; 16 rows 11 | 25; 64 rows - | 35 | 193
// 3 bits take 4 to 10 % longer, 4 bits 15 to 40 %.
inline RowsPlan plan_packed(int64_t rows, int64_t groups, int O, int blocks, bool tight) {
  const double each = (double)rows / std::min(rows, groups);   // rows of a group
  const int slabs = 2 * blocks, few_waves = std::min(blocks, kFewWaves);
  const TileCost large[] = {{256, 256, 3, 1.4, 1.65}, {128, 256, 2, 1.0, 1.15}, {64, 256, 1.5, 0.72, 0.95}};
  const TileCost shared[] = {{64, 64, 1, each <= 16 ? 0.07 : each <= 32 ? 0.095 : 0.15,
                              each <= 16 ? 0.09 : each <= 32 ? 0.12 : 0.2}};
  double best = 1e30;
  if (!tight) {
    // x from any address (2 bits; 16 x 16 shared | 128 rows by workgroups):
    //   I 4096, O 4096: 1 row 8 | 83; 64 rows 25 | 83; 256 rows 90 | 85; 2001 rows 683 | 99 (aligned 81); 4096 rows
    //     1386 | 184
    //   I 4096, O 14336: 64 rows 78 | 84; 512 rows 611 | 97.  I 14336, O 4096: 1 row 18 | 267; 256 rows 246 | 295
    // (3 bits 2 to 8 % longer, 4 bits 5 to 25 %), and 64 groups of 2048 x 7168, super-blocks, where each group with rows
    // has a panel: 128 rows 342 | 408, 512 rows 350 | 377, 1024 rows 364 | 378, 2048 rows 666 | 384
    const TileCost few[] = {{16, 16, 0.7, 0.04, 0.068}};
    const TileCost loose[] = {{128, 256, 2, 1.2, 1.42}};
    const RowsPlan plan = cheapest(rows, groups, O, slabs, few, true, few_waves, best, RowsPlan{});
    return cheapest(rows, groups, O, slabs, loose, false, kRingWaves, best, plan, (double)std::min(rows, groups));
  }
  const TileCost few[] = {{16, 16, 0.7, 0.02, 0.03}};
  RowsPlan plan = cheapest(rows, groups, O, slabs, few, true, few_waves, best, RowsPlan{});
  plan = cheapest(rows, groups, O, slabs, shared, true, std::min(blocks, kSplitWaves), best, plan);
  return cheapest(rows, groups, O, slabs, large, false, kRingWaves, best, plan);
}

// hidden and dhidden of the adapters: rows times a matrix of `rank` columns by wavefronts that share the sum, at the
// costs of plan_rows, which were fitted there to eight of them; tiles of 16 x 16 have up to sixteen here.  (Those are taken
// only where they number far fewer than a launch of sixteen wavefronts holds: of more rows 64 x 16 is cheaper, of a rank
// beyond 16 16 x 64.)
inline RowsPlan plan_adapter(int64_t rows, int64_t segments, int rank, int slabs, bool tight) {
  const TileCost aligned[] = {{64, 64, 1, 0.165, 0.22}, {64, 16, 1, 0.1, 0.115}, {16, 64, 1, 0.06, 0.1}, {16, 16, 0.5, 0.02, 0.055}};
  const TileCost loose[] = {{64, 64, 1, 0.17, 0.42}, {64, 16, 1, 0.1, 0.21}, {16, 64, 1, 0.07, 0.15}, {16, 16, 0.5, 0.025, 0.08}};
  double best = 1e30;
  return cheapest(rows, segments, rank, slabs, tight ? aligned : loose, true, std::min(slabs, kSplitWaves), best, RowsPlan{});
}

// y and dx from hidden: no steps: panels of 16 rows and 256 columns, for segments of 16 rows and fewer; else panels of 64
// rows and `steps` times 64 columns, such that whole rounds of 1024 workgroups (four on each of 256 CUs) with a start as
// long as three steps take least.
struct UpPlan {
  int steps;
  int64_t blocks;
};
inline UpPlan plan_adapter_up(int64_t rows, int64_t segments, int cols) {
  if (rows <= 16 * segments) return {0, most_panels(rows, segments, 16) * tiles_of(cols, 256)};
  const int64_t all = tiles_of(cols, 64), panels = rows / 64 + (std::min(rows, segments) + 1) / 2;
  int64_t best = INT64_MAX;
  int steps = 1;
  for (int n = 1; n <= 32; ++n) {
    const int64_t cost = tiles_of(panels * tiles_of(all, n), 1024) * (n + 3);
    if (cost < best) {
      best = cost;
      steps = n;
    }
  }
  return {steps, most_panels(rows, segments, 64) * tiles_of(all, steps)};
}

// Wavefronts that share the sums of dA and dB: half as many again as an adapter has pairs of slabs of 32
// rows on average.
inline int plan_adapter_weights(int64_t rows, int64_t segments, int64_t adapters) {
  const int64_t slabs = most_panels(rows, segments, 64) * 3 / 2;
  return (int)std::max<int64_t>(1, std::min<int64_t>(kSplitWaves, (slabs + adapters - 1) / adapters));
}

// How a sum over rows is cut: tiles of `size` x `size`.  Where nothing fits a launch, one that does not.
struct SumsPlan {
  bool split;
  int size, waves;
};

// Tiles of the sums of all groups; of H those on and above the diagonal, two rows of them taken as one.
inline int64_t sum_tiles(int64_t groups, int O, int I, bool gram, int size) {
  const int64_t tm = tiles_of(O, size), tn = tiles_of(I, size);
  return groups * (gram ? (tn + 1) / 2 * (tn + 1) : tm * tn);
}

// dW, and H (gram): whole workgroups on 256 x 256 or 128 x 128 tiles, or wavefronts that share the sum of 64 x 64 or
// 32 x 32 ones: the cheapest by a tile's start and slabs, fitted to dW of one group (us, 256 | 128 | 64 | 32):
//   256 x 256: 4096 rows 96 | - | 14 | 8; 16384 rows 318 | - | 49 | 42
//   1024 x 1024: 4096 rows 95 | 34 | 19 | 38; 16384 rows 319 | 121 | 62 | 177
//   2048 x 2048: 256 rows 21 | 8 | 12 | 14; 4096 rows 96 | 42 | 61 | 137; 16384 rows 318 | 133 | 304 | 850
//   4096 x 4096: 64 rows - | 17 | 18 | -; 256 rows 21 | 19 | 38 | 46; 4096 rows 105 | 120 | 235 | 514; 16384 rows
//     401 | 527 | 1451 | -
//   8192 x 8192: 256 rows 72 | 66 | 138 | 170; 4096 rows 432 | 475 | 883 | 2120; 16384 rows 1607 | 2516 | - | -
// and H, which stores most tiles twice: 4096 x 4096 from 1024 rows 57 | 39 | 57 | 83, 8192 x 8192 from 64 rows
// - | 59 | 51 | -, 1024 rows 156 | 106 | 202 | 306, 16384 rows 1093 | 1857 | - | -; with whole tiles | what the rule takes:
// 2048 x 2048 from 8192 rows 180 | 69, 4096 x 4096 from 4096 120 | 100, 8192 202 | 181, 12288 278 | 259, 6144 x 6144
// from 8192 392 | 348, 8192 x 8192 from 4096 348 | 319; 5120 x 5120 from 8192 209 | 218, the one that it misses.
inline SumsPlan plan_sums(int64_t rows, int64_t groups, int O, int I, bool tight, bool gram) {
  const double slabs = (double)rows / 64 / groups;
  const int waves = (int)std::max<int64_t>(1, std::min<int64_t>(kSplitWaves, tiles_of(rows, 64)));
  const auto cost = [&](int size, double start, double more_start, double alone, double full) {
    const int64_t tiles = sum_tiles(groups, O, I, gram, size);
    if (!fits_launch(tiles, 64 * (size < 128 ? waves : kRingWaves))) return 1e30;
    const double rounds = tiles / 256.0, load = std::min(1.0, rounds);
    const double whole = groups == 1 && size != 128 ? std::ceil(rounds) : rounds;
    return std::max(1.0, whole) * (start + more_start * load + (slabs + 0.5) * (alone + (full - alone) * load));
  };
  const double far = slabs > 100 ? 1.25 : 1;   // what the L2 holds of a long sum's operands no longer serves small tiles
  const double us_whole = !tight ? 1e30 : cost(256, gram ? 20 : 9, gram ? 12 : 3.5, 1.2, gram ? 1.35 : 1.5);
  const double us_quarter = cost(128, gram ? 6.5 : 2, 0, 0.45 * far, 0.5 * far);
  const double us_64 = cost(64, gram ? 1.4 : 0.7, 0, 0.17, 0.23), us_32 = cost(32, gram ? 0.3 : 0.15, 0, 0.08, 0.14);
  const double us_split = std::min(us_64, us_32);
  if (us_whole < std::min(us_quarter, us_split)) return {false, 256, kRingWaves};
  if (us_quarter < us_split) return {false, 128, kRingWaves};
  return {true, us_32 < us_64 ? 32 : 64, waves};
}

// How ids are brought into order: by one workgroup, or chunk by chunk, of which there are at most 128, so that a
// workgroup counts over all of them itself.  The chunks' counts, kept in the ids' places until these are known, take less
// than a quarter of them and one chunk's: about half at most, with two chunks of which the second is short.  `waves`
// wavefronts count, with a histogram each in LDS (64 KB in all).
struct OrderPlan {
  int threads, waves, chunks;
  int64_t chunk;
};
inline OrderPlan plan_order(int64_t count, int groups) {
  constexpr int kWords = 15360;
  const int64_t chunk = std::max({(int64_t)1024, (int64_t)4 * groups, tiles_of(tiles_of(count, 128), 64) * 64});
  if (count <= std::max((int64_t)8192, chunk)) {
    const int waves = (int)std::min<int64_t>({16, kWords / groups - 1, tiles_of(count, 64)});
    return {std::max(64 * waves, groups > 256 ? 1024 : 256), waves, 1, count};
  }
  return {512, std::min(8, kWords / groups), (int)tiles_of(count, chunk), chunk};
}

}  // namespace gsq
