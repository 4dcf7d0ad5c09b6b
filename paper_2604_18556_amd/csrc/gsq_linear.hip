// The packed layer in use: its bytes laid out for the matrix instructions, and the product of grouped
// rows with it.
#include <hip/hip_runtime.h>

#include <algorithm>

#include "gsq_split.hpp"

namespace gsq {
namespace {

// Where code j (0 .. 31) of a lane is kept in its `bits` words.  Four codes that are neighbours lie at
// the same place in the four bytes of a word, so that one mask takes out four byte-wide indices:
//   1 bit:  bit 8 (j % 4) + j / 4
//   2 bits: word j / 16, bits 8 (j % 4) + 2 (j / 4 % 4)
//   3 bits: the lower two as for 2 bits, the third in word 2 as for 1 bit
//   4 bits: word j / 8, bits 8 (j % 4) + 4 (j / 4 % 2)
__device__ __forceinline__ void place_code(uint32_t* words, int bits, int j, uint32_t code) {
  const int byte = 8 * (j & 3), quad = j >> 2;
  if (bits == 1) {
    words[0] |= code << (byte + quad);
  } else if (bits == 4) {
    words[quad >> 1] |= code << (byte + 4 * (quad & 1));
  } else {
    words[quad >> 2] |= (code & 3) << (byte + 2 * (quad & 3));
    if (bits == 3) words[2] |= (code >> 2) << (byte + quad);
  }
}
// A field of at most 8 bits from little-endian bits; the next byte is read only if the field reaches it.
__device__ __forceinline__ uint32_t bit_field(const uint8_t* p, int64_t bit, int width) {
  const int64_t at = bit >> 3;
  const int shift = (int)(bit & 7);
  uint32_t v = p[at] >> shift;
  if (shift + width > 8) v |= (uint32_t)p[at + 1] << (8 - shift);
  return v & ((1u << width) - 1);
}

// Code of weight w (its index over all layers) in the packed bytes.
__device__ __forceinline__ uint32_t packed_code(const uint8_t* p, int layout, int bits, int64_t w) {
  if (layout == GSQ_LAYOUT_SUPERBLOCK) return bit_field(p + (w >> 8) * 110 + 14, (w & 255) * 3, 3);
  if (layout == GSQ_LAYOUT_BASE3) {
    uint32_t v = p[w / 5];
    for (int j = (int)(w % 5); j; --j) v /= 3;
    return v % 3;
  }
  return bit_field(p, w * bits, bits);
}

__device__ __forceinline__ uint16_t two_bytes(const uint8_t* p) { return p[0] | (uint16_t)(p[1] << 8); }

// A thread's elements of `count`, with unpack_blocks() workgroups.
template <class F>
__device__ __forceinline__ void each_of(int64_t count, F f) {
  for (int64_t at = (int64_t)blockIdx.x * 256 + threadIdx.x; at < count; at += (int64_t)gridDim.x * 256) f(at);
}

// A lane of a unit: its 32 codes.
__device__ __forceinline__ void unpack_codes(const uint8_t* packed, int layout, int packed_bits, const PackedLayer& L,
                                             int64_t at, uint32_t* codes) {
  const int lane = (int)(at & 63);
  const int64_t unit = at >> 6;
  const int kb = (int)(unit % L.blocks);
  const int64_t tile = unit / L.blocks;
  const int64_t e = tile / L.tiles;
  const int64_t o = (tile % L.tiles) * 16 + (lane & 15), i0 = (int64_t)kb * 128 + (lane >> 4) * 32;
  uint32_t words[4] = {0, 0, 0, 0};
  if (o < L.O)
    for (int j = 0; j < 32 && i0 + j < L.I; ++j) {
      const uint32_t c = packed_code(packed, layout, packed_bits, (e * L.O + o) * L.I + i0 + j);
      place_code(words, L.bits, j, min(c, (uint32_t)L.n_levels - 1));
    }
  for (int k = 0; k < L.bits; ++k) codes[at * L.bits + k] = words[k];
}
__global__ __launch_bounds__(256) void k_unpack_codes(const uint8_t* __restrict__ packed, int layout,
                                                      int packed_bits, PackedLayer L, int64_t lanes,
                                                      uint32_t* __restrict__ codes) {
  each_of(lanes, [&](int64_t at) { unpack_codes(packed, layout, packed_bits, L, at, codes); });
}

// Where the scale of channel n of a tile and inputs 16 j .. is kept: for groups of 16 with the unit's lanes,
// the two of a lane side by side; else by group, 16 channels side by side.
__device__ __forceinline__ void place_of_scale(const PackedLayer& L, bool fine, int64_t at, int64_t& tile, int& n,
                                               int& group) {
  if (fine) {
    const int64_t unit = at >> 7;
    const int lane = (int)(at >> 1) & 63;
    tile = unit / L.blocks;
    n = lane & 15;
    group = (int)(unit % L.blocks) * 8 + (lane >> 4) * 2 + (int)(at & 1);
  } else {
    tile = at / 16 / L.scale_groups;
    n = (int)(at & 15);
    group = (int)(at / 16 % L.scale_groups);
  }
}

// The kept scales, zero where there is no channel or group.
__global__ __launch_bounds__(256) void k_unpack_scales(const uint8_t* __restrict__ packed, int layout,
                                                       PackedLayer L, int64_t at_byte, int64_t count,
                                                       uint16_t* __restrict__ scales) {
  each_of(count, [&](int64_t at) {
    int64_t tile;
    int n, g;
    place_of_scale(L, L.gs == 16, at, tile, n, g);
    const int64_t e = tile / L.tiles, o = (tile % L.tiles) * 16 + n;
    uint16_t v = 0;
    if (o < L.O && g < L.I / L.gs) {
      const int64_t k = (e * L.O + o) * (L.I / L.gs) + g;
      v = two_bytes(layout == GSQ_LAYOUT_SUPERBLOCK ? packed + k * 110 : packed + at_byte + 2 * k);
    }
    scales[at] = v;
  });
}

__global__ __launch_bounds__(256) void k_unpack_sub(const uint8_t* __restrict__ packed, PackedLayer L,
                                                    int64_t count, uint8_t* __restrict__ sub) {
  each_of(count, [&](int64_t at) {
    int64_t tile;
    int n, g;
    place_of_scale(L, true, at, tile, n, g);
    const int64_t e = tile / L.tiles, o = (tile % L.tiles) * 16 + n;
    uint32_t v = 0;
    if (o < L.O && g < L.I / 16) {
      const int64_t rec = (e * L.O + o) * (L.I / 256) + g / 16;
      v = bit_field(packed + rec * 110 + 2, (g & 15) * 6, 6);
    }
    sub[at] = (uint8_t)v;
  });
}

// scale * level rounded to fp32, for a second rounding to the type of x.  The empty asm keeps the compiler
// from joining product and conversion into one instruction, which would round once.
__device__ __forceinline__ float scaled_level(float scale, float level) {
  float p = scale * level;
  asm("" : "+v"(p));
  return p;
}

// ---- from codes to weights.  Scales of one group of inputs give a table of all 2^BITS weights; a lane's
// codes pick from it.  v_perm_b32 picks four bytes of eight by four selectors, so the table is kept as its low
// bytes and its high bytes, four codes are four selectors, and two more picks put the bytes together:
// 1.5 instructions per weight at 2 bits, 2 at 3 bits, 3.3 at 4 bits.
template <class T, int BITS>
struct WeightTable {
  static constexpr int N = 1 << BITS, WORDS = (N + 3) / 4;
  uint32_t lo[WORDS], hi[WORDS];

  static __device__ __forceinline__ uint32_t pair(float a, float b) {
    typedef float f32x2 __attribute__((ext_vector_type(2)));
    typedef typename T::elem e2 __attribute__((ext_vector_type(2)));
    return __builtin_bit_cast(uint32_t, __builtin_convertvector((f32x2{a, b}), e2));
  }
  __device__ __forceinline__ WeightTable(float scale, const float* levels) {
#pragma unroll
    for (int w = 0; w < WORDS; ++w) {
      float v[4];
#pragma unroll
      for (int k = 0; k < 4; ++k) v[k] = 4 * w + k < N ? scaled_level(scale, levels[4 * w + k]) : 0.f;
      const uint32_t p01 = pair(v[0], v[1]), p23 = N > 2 ? pair(v[2], v[3]) : 0;
      lo[w] = __builtin_amdgcn_perm(p23, p01, 0x06040200);
      hi[w] = __builtin_amdgcn_perm(p23, p01, 0x07050301);
    }
  }
  // Weights 4 q .. 4 q + 3 of a lane's 32 as two words.
  __device__ __forceinline__ void pick(const uint32_t* words, int q, uint32_t& d0, uint32_t& d1) const {
    uint32_t l, h;
    if constexpr (BITS == 1) {
      const uint32_t sel = words[0] >> q & 0x01010101u;
      l = __builtin_amdgcn_perm(hi[0], lo[0], sel);
      h = __builtin_amdgcn_perm(lo[0], hi[0], sel);
    } else if constexpr (BITS == 2) {
      const uint32_t sel = words[q >> 2] >> (2 * (q & 3)) & 0x03030303u;
      l = __builtin_amdgcn_perm(hi[0], lo[0], sel);
      h = __builtin_amdgcn_perm(lo[0], hi[0], sel);
    } else if constexpr (BITS == 3) {
      const uint32_t top = q < 2 ? words[2] << (2 - q) : words[2] >> (q - 2);
      const uint32_t sel = (words[q >> 2] >> (2 * (q & 3)) & 0x03030303u) | (top & 0x04040404u);
      l = __builtin_amdgcn_perm(lo[1], lo[0], sel);
      h = __builtin_amdgcn_perm(hi[1], hi[0], sel);
    } else {
      const uint32_t nibbles = words[q >> 1] >> (4 * (q & 1));
      const uint32_t sel = nibbles & 0x07070707u;
      // selectors 12 and 13 give 0 and 255: the mask of the upper eight
      const uint32_t mask = __builtin_amdgcn_perm(0, 0, (nibbles >> 3 & 0x01010101u) | 0x0c0c0c0cu);
      const uint32_t l0 = __builtin_amdgcn_perm(lo[1], lo[0], sel), l1 = __builtin_amdgcn_perm(lo[3], lo[2], sel);
      const uint32_t h0 = __builtin_amdgcn_perm(hi[1], hi[0], sel), h1 = __builtin_amdgcn_perm(hi[3], hi[2], sel);
      l = (l1 & mask) | (l0 & ~mask);
      h = (h1 & mask) | (h0 & ~mask);
    }
    d0 = __builtin_amdgcn_perm(h, l, 0x05010400);
    d1 = __builtin_amdgcn_perm(h, l, 0x07030602);
  }
  // Weights 8 s .. 8 s + 7.
  __device__ __forceinline__ typename T::frag frag(const uint32_t* words, int s) const {
    union { uint32_t d[4]; typename T::frag f; } w;
    pick(words, 2 * s, w.d[0], w.d[1]);
    pick(words, 2 * s + 1, w.d[2], w.d[3]);
    return w.f;
  }
};

// What one lane holds of a unit: its 32 codes, and the scales of their first and second half.
template <int BITS, bool kFine>
struct LaneCodes {
  uint32_t words[BITS];
  uint32_t scales;          // fp16: one, or two for groups of 16 (kFine); sub-block scales: two bytes
  uint32_t d;               // SUPERBLOCK: fp16

  // of lane slot `slot` (16 g + n) of unit (tile, kb)
  __device__ __forceinline__ void load(const PackedLayer& L, int64_t tile, int kb, int slot) {
    const int64_t unit = tile * L.blocks + kb;
    const uint32_t* p = L.codes + (unit * 64 + slot) * BITS;
#pragma unroll
    for (int k = 0; k < BITS; ++k) words[k] = p[k];
    d = 0;
    if constexpr (kFine) {
      if (L.sub) {
        scales = reinterpret_cast<const uint16_t*>(L.sub)[unit * 64 + slot];
        d = L.scales[(tile * L.scale_groups + (kb >> 1)) * 16 + (slot & 15)];
      } else {
        scales = reinterpret_cast<const uint32_t*>(L.scales)[unit * 64 + slot];
      }
    } else {
      const int group = (kb * 128 + (slot >> 4) * 32) / L.gs;
      scales = L.scales[(tile * L.scale_groups + group) * 16 + (slot & 15)];
    }
  }
  __device__ __forceinline__ void arrived() {
#pragma unroll
    for (int k = 0; k < BITS; ++k) asm volatile("" : "+v"(words[k]));
    asm volatile("" : "+v"(scales), "+v"(d));
  }
  __device__ __forceinline__ float scale(const PackedLayer& L, int half) const {
    const auto f16 = [](uint32_t v) { return (float)__builtin_bit_cast(_Float16, (uint16_t)v); };
    if constexpr (!kFine) return f16(scales);
    if (L.sub) return f16(d) * (float)(half ? scales >> 8 : scales & 255);
    return f16(half ? scales >> 16 : scales);
  }
};

// ---- few rows, or too few tiles for whole workgroups: COLS channels and up to 64 rows, the units shared by the
// wavefronts as tile_split() does it.  x goes through LDS, the weights from the codes to registers.
//
// At one row bound by latency, with one unit of codes in flight for each wavefront: 4096 x 14336 (23 MB) in 11.3 us,
// 4096 x 4096 in 6.1, vector units busy 0.36 of the time (some three instructions for a weight of 3 bits) and wavefronts
// waiting 0.46.  x straight from memory to the fragments, without LDS: 12.8
// us at one row, and 23 at 16 instead of 13.
template <class T, int BITS, bool kFine, int COLS, int TM, bool kLoose>
__device__ __forceinline__ void packed_shared(const PackedLayer& L, const typename T::elem* x, typename T::elem* y,
                                              int group, int64_t first, int ms, int n0, int vector_out, uint8_t* smem) {
  using E = typename T::elem;
  constexpr int MI = TM / 16, NJ = COLS / 16, A_SLAB = TM * ROW_BYTES, OWN = 2 * A_SLAB;
  static_assert(TM * COLS * 4 <= OWN, "the sums take the slabs' place");
  using Slab = std::conditional_t<kLoose, LooseAlong<E, TM>, Copied<SlabAlong<TM, TM / 8>>>;
  const int lane = threadIdx.x & 63, waves = blockDim.x >> 6, g = lane >> 4;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  uint8_t* const own = smem + wave * OWN;
  const auto slab_of_x = [&] {
    if constexpr (kLoose)
      return Slab(x + first * L.I, L.I, ms, L.I, 0);
    else
      return Slab(x + first * L.I, (int64_t)L.I * 2, ms, 0, lane);
  };
  Slab a[2] = {slab_of_x(), slab_of_x()};   // the two of a unit
  const int64_t tile0 = (int64_t)group * L.tiles;
  int64_t tile[NJ];
  LaneCodes<BITS, kFine> next[NJ];
  f32x4 acc[MI][NJ] = {};
  const auto fetch = [&](int kb) {
    a[0].fetch(2 * kb, own);
    a[1].fetch(2 * kb + 1, own + A_SLAB);
#pragma unroll
    for (int j = 0; j < NJ; ++j) next[j].load(L, tile[j], kb, lane);
  };
#pragma unroll
  for (int j = 0; j < NJ; ++j) tile[j] = tile0 + min(n0 / 16 + j, L.tiles - 1);   // beyond: not stored
  if (wave < L.blocks) fetch(wave);
  for (int kb = wave; kb < L.blocks; kb += waves) {
    a[0].commit(own);
    a[1].commit(own + A_SLAB);
    wait_all();
    typename T::frag fa[MI][4];
#pragma unroll
    for (int i = 0; i < MI; ++i)
#pragma unroll
      for (int s = 0; s < 4; ++s)   // inputs 32 g + 8 s of the unit
        fa[i][s] = read_frag<typename T::frag>(own + (g >> 1) * A_SLAB, i * 16 + (lane & 15), 4 * (g & 1) + s);
    LaneCodes<BITS, kFine> now[NJ];
#pragma unroll
    for (int j = 0; j < NJ; ++j) now[j] = next[j];
    wait_reads();
    if (kb + waves < L.blocks) fetch(kb + waves);
#pragma unroll
    for (int j = 0; j < NJ; ++j)
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        const WeightTable<T, BITS> table(now[j].scale(L, kFine ? h : 0), L.levels);
#pragma unroll
        for (int s = 2 * h; s < 2 * h + 2; ++s) {
          const typename T::frag w = table.frag(now[j].words, s);
#pragma unroll
          for (int i = 0; i < MI; ++i) acc[i][j] = T::mfma(w, fa[i][s], acc[i][j]);
        }
      }
  }
  split_sums<TM, COLS>(acc, own);
  const ResultColumns<E> out{y + first * L.O + n0, L.O, ms, L.O - n0, vector_out != 0};
  store_added<TM, COLS, f32x4>(smem, OWN, min(waves, L.blocks), out, false, out);
}

// Panels of 64 rows, of which the shorter ones are taken as 32 or 16; with 16 channels, panels of 16.
template <int COLS>
constexpr int shared_panel() { return COLS == 16 ? 16 : 64; }
template <int COLS>
constexpr int shared_waves() { return COLS == 16 ? kFewWaves : kSplitWaves; }

template <class T, int BITS, bool kFine, int COLS, bool kLoose>
__global__ __launch_bounds__(64 * shared_waves<COLS>()) void k_packed_shared(PackedLayer L, GroupRows rows,
                                                                            const typename T::elem* __restrict__ x,
                                                                            typename T::elem* __restrict__ y, int vector_out) {
  extern __shared__ __attribute__((aligned(16))) uint8_t smem[];
  constexpr int TM = shared_panel<COLS>();
  const int tiles_n = (L.O + COLS - 1) / COLS;
  PanelPlace at;
  if (!find_panel(rows, TM, blockIdx.x / (unsigned)tiles_n, at)) return;
  int tm, tn;
  tile_at(lin_of((int)(blockIdx.x - at.before * tiles_n), at.panels * tiles_n), at.panels, tiles_n, tm, tn);
  const int64_t first = at.first + (int64_t)tm * TM;
  const int ms = (int)min(at.end - first, (int64_t)TM);
  if constexpr (COLS == 64) {
    if (ms > 32)
      return packed_shared<T, BITS, kFine, COLS, 64, kLoose>(L, x, y, at.group, first, ms, tn * COLS, vector_out, smem);
    if (ms > 16)
      return packed_shared<T, BITS, kFine, COLS, 32, kLoose>(L, x, y, at.group, first, ms, tn * COLS, vector_out, smem);
  }
  packed_shared<T, BITS, kFine, COLS, 16, kLoose>(L, x, y, at.group, first, ms, tn * COLS, vector_out, smem);
}

// ---- many rows: tiles as for a dense layer, whose slabs of weights the wavefronts write to LDS from the
// codes.  Half a unit's inputs (64) make a slab.  A wavefront writes a quarter of it: lane 32 j + 16 h + n the
// 32 weights of channel n, tile 2 i + j, lane slot (2 (k % 2) + h, n), for i = 0 .. in turn.
template <class T, int BITS, bool kFine, int ROWS>
struct SlabPacked {
  static constexpr bool kCopied = false;
  static constexpr int LOADS = ROWS / 32, UNITS = LOADS / 4;
  const PackedLayer& L;
  int64_t tile0;             // first tile of the group
  int tile[UNITS];
  LaneCodes<BITS, kFine> codes[UNITS];
  WeightTable<T, BITS> table;

  __device__ __forceinline__ SlabPacked(const PackedLayer& L_, int group, int n0, int wave, int lane)
      : L(L_), tile0((int64_t)group * L_.tiles), table(0.f, L_.levels) {
#pragma unroll
    for (int i = 0; i < UNITS; ++i)   // channels beyond the last are not stored
      tile[i] = min(n0 / 16 + wave * (ROWS / 64) + 2 * i + (lane >> 5), L.tiles - 1);
  }
  __device__ __forceinline__ void prefetch(int k) {
    const int lane = threadIdx.x & 63, kb = k >> 1;
    const int slot = (2 * (k & 1) + ((lane >> 4) & 1)) * 16 + (lane & 15);
#pragma unroll
    for (int i = 0; i < UNITS; ++i) codes[i].load(L, tile0 + tile[i], min(kb, L.blocks - 1), slot);
  }
  // eight weights of each lane into slab k; with the last of them, the codes of slab k + 1 are fetched
  template <bool kEnd>
  __device__ __forceinline__ void load(int k, int j, uint8_t* lds) {
    const int lane = threadIdx.x & 63, i = j / 4, s = j % 4;
    if (j == 0)   // the codes are waited for here, not where a table might be begun early
#pragma unroll
      for (int u = 0; u < UNITS; ++u) codes[u].arrived();
    if (s == 0 || (kFine && s == 2))   // slabs past the last unit are zeros
      table = WeightTable<T, BITS>(!kEnd || k >> 1 < L.blocks ? codes[i].scale(L, s / 2) : 0.f, L.levels);
    const i32x4 w = __builtin_bit_cast(i32x4, table.frag(codes[i].words, s));
    const int row = (2 * i + (lane >> 5)) * 16 + (lane & 15), chunk = 4 * ((lane >> 4) & 1) + s;
    *reinterpret_cast<i32x4*>(lds + row * ROW_BYTES + ((chunk ^ swz(row)) << 4)) = w;
    if (j == LOADS - 1) prefetch(k + 1);
  }
  static __device__ __forceinline__ i32x4 frag(const uint8_t* slab, int row0, int half, int lane) {
    return read_frag<i32x4>(slab, row0 + (lane & 15), half * 4 + (lane >> 4));
  }
};

template <class T, int BITS, bool kFine, class S, bool kLoose>
__device__ __forceinline__ void packed_tile(const PackedLayer& L, const typename T::elem* x, typename T::elem* y,
                                            const RowsTile& at, int vector_out, uint8_t* smem) {
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  SlabPacked<T, BITS, kFine, S::TN> b(L, at.group, at.n0, wave, lane);
  typename T::acc acc[S::MI][S::NJ];
  if constexpr (kLoose) {
    RingLoose<LooseAlong<typename T::elem, S::TM, S::TM / 32>> a(x + at.first * L.I, L.I, at.ms, L.I, wave);
    tile_ring<T, S>(a, b, (L.I + 63) / 64, acc, smem);
  } else {
    SlabAlong<S::TM, S::TM / 32, true> a(x + at.first * L.I, (int64_t)L.I * 2, at.ms, wave, lane);
    tile_ring<T, S>(a, b, (L.I + 63) / 64, acc, smem);
  }
  const ResultColumns<typename T::elem> out{y + at.first * L.O + at.n0, L.O, at.ms, L.O - at.n0, vector_out != 0};
  tile_results<S>(acc, smem, out, false, out);
}

template <class T, int BITS, bool kFine>
__global__ __launch_bounds__(256, 1) void k_packed_tile(PackedLayer L, GroupRows rows,
                                                        const typename T::elem* __restrict__ x,
                                                        typename T::elem* __restrict__ y, int height, int vector_out) {
  extern __shared__ __attribute__((aligned(16))) uint8_t smem[];
  RowsTile at;
  if (!find_rows_tile(rows, height, Whole::TN, L.O, at)) return;
  if (at.ms > Half::TM)
    packed_tile<T, BITS, kFine, Whole, false>(L, x, y, at, vector_out, smem);
  else if (at.ms > Low::TM)
    packed_tile<T, BITS, kFine, Half, false>(L, x, y, at, vector_out, smem);
  else
    packed_tile<T, BITS, kFine, Low, false>(L, x, y, at, vector_out, smem);
}

// x from any address, by way of registers: 2001 rows through 4096 x 4096 at 2 bits in 99 us (aligned: 81).
template <class T, int BITS, bool kFine>
__global__ __launch_bounds__(256, 1) void k_packed_loose(PackedLayer L, GroupRows rows,
                                                         const typename T::elem* __restrict__ x,
                                                         typename T::elem* __restrict__ y, int vector_out) {
  extern __shared__ __attribute__((aligned(16))) uint8_t smem[];
  RowsTile at;
  if (find_rows_tile(rows, Half::TM, Half::TN, L.O, at))
    packed_tile<T, BITS, kFine, Half, true>(L, x, y, at, vector_out, smem);
}

}  // namespace

hipError_t launch_unpack_layer(const gsq_config& cfg, const uint8_t* packed, const PackedLayer& L,
                               hipStream_t s) {
  const int64_t tiles = (int64_t)cfg.batch * L.tiles, weights = (int64_t)cfg.batch * L.O * L.I;
  const int packed_bits = cfg.layout == GSQ_LAYOUT_SUPERBLOCK ? 3 : L.bits;
  const int64_t lanes = tiles * L.blocks * 64;
  const int64_t scales = tiles * (L.gs == 16 ? (int64_t)L.blocks * 128 : (int64_t)L.scale_groups * 16);
  k_unpack_codes<<<unpack_blocks(lanes), 256, 0, s>>>(packed, cfg.layout, packed_bits, L, lanes,
                                                      const_cast<uint32_t*>(L.codes));
  hipError_t e = hipGetLastError();
  if (e != hipSuccess) return e;
  const int64_t at_byte = cfg.layout == GSQ_LAYOUT_BASE3 ? (weights + 4) / 5 : weights * packed_bits / 8;
  k_unpack_scales<<<unpack_blocks(scales), 256, 0, s>>>(packed, cfg.layout, L, at_byte, scales,
                                                        const_cast<uint16_t*>(L.scales));
  e = hipGetLastError();
  if (e != hipSuccess || !L.sub) return e;
  k_unpack_sub<<<unpack_blocks(lanes * 2), 256, 0, s>>>(packed, L, lanes * 2, const_cast<uint8_t*>(L.sub));
  return hipGetLastError();
}

namespace {

template <class T, int BITS, bool kFine, int COLS, bool kLoose>
hipError_t launch_shared(const PackedLayer& L, const GroupRows& rows, const typename T::elem* x, typename T::elem* y,
                         int vector_out, hipStream_t s) {
  constexpr int TM = shared_panel<COLS>();
  const int waves = std::min(shared_waves<COLS>(), L.blocks);
  return launch_lds<k_packed_shared<T, BITS, kFine, COLS, kLoose>>(most_panels(rows, TM) * tiles_of(L.O, COLS), 64 * waves,
                                                                   (size_t)waves * 2 * TM * ROW_BYTES, s, L, rows, x, y,
                                                                   vector_out);
}

template <class T, int BITS, bool kFine>
hipError_t launch_packed(const PackedLayer& L, const GroupRows& rows, const void* x, void* y, hipStream_t s) {
  using E = typename T::elem;
  const int vector_out = four_at_once(y, T::kDtype, L.O);
  const E* xe = static_cast<const E*>(x);
  E* ye = static_cast<E*>(y);
  const bool tight = aligned16(x);
  const RowsPlan plan = plan_packed(rows.rows, rows.groups, L.O, L.blocks, tight);
  if (!plan.height) return hipErrorInvalidConfiguration;
  const int64_t tiles = most_panels(rows, plan.height) * tiles_of(L.O, plan.width);
  if (!plan.split)
    return tight ? launch_ring<k_packed_tile<T, BITS, kFine>>(tiles, s, L, rows, xe, ye, plan.height, vector_out)
                 : launch_ring<k_packed_loose<T, BITS, kFine>>(tiles, s, L, rows, xe, ye, vector_out);
  if (plan.height == 64) return launch_shared<T, BITS, kFine, 64, false>(L, rows, xe, ye, vector_out, s);
  return tight ? launch_shared<T, BITS, kFine, 16, false>(L, rows, xe, ye, vector_out, s)
               : launch_shared<T, BITS, kFine, 16, true>(L, rows, xe, ye, vector_out, s);
}

template <class T, int BITS>
hipError_t launch_packed(const PackedLayer& L, const GroupRows& rows, const void* x, void* y, hipStream_t s) {
  return L.sub || L.gs == 16 ? launch_packed<T, BITS, true>(L, rows, x, y, s)
                             : launch_packed<T, BITS, false>(L, rows, x, y, s);
}

template <class T>
hipError_t launch_packed(const PackedLayer& L, const GroupRows& rows, const void* x, void* y, hipStream_t s) {
  switch (L.bits) {
    case 1: return launch_packed<T, 1>(L, rows, x, y, s);
    case 2: return launch_packed<T, 2>(L, rows, x, y, s);
    case 3: return launch_packed<T, 3>(L, rows, x, y, s);
    default: return launch_packed<T, 4>(L, rows, x, y, s);
  }
}

}  // namespace

hipError_t launch_packed_product(const PackedLayer& L, int dtype, const GroupRows& rows, const void* x,
                                 void* y, hipStream_t s) {
  if (rows.rows == 0) return hipSuccess;
  return dtype == GSQ_DT_BF16 ? launch_packed<Bf16>(L, rows, x, y, s) : launch_packed<F16>(L, rows, x, y, s);
}

}  // namespace gsq
