// The product of a small output tile by wavefronts that share the sum between them: each takes a part of k
// for the whole tile, with slabs of its own in LDS, and the partial sums are added in a fixed order.
//
// For products with too few tiles of 256 x 256 for the GPU, and for operands that are not aligned to 16
// bytes.  No wavefront waits for another until the end.
#pragma once
#include <hip/hip_runtime.h>
#include <stdint.h>

#include "gsq_tile.hpp"

namespace gsq {
namespace {

// 16 bytes from any address, of which the first n (<= 16 / sizeof(E)) elements are in bounds and the others
// become zero.
template <class E>
__device__ __forceinline__ i32x4 load_chunk(const E* p, int n) {
  constexpr int PER = 16 / (int)sizeof(E);
  i32x4 v = {0, 0, 0, 0};
  if (n >= PER) {
    __builtin_memcpy(&v, p, 16);
  } else if (n > 0) {
    // eight, four, two bytes and one, of which n's bits say which there are
    uint64_t part[2] = {0, 0};
    const uint8_t* b = reinterpret_cast<const uint8_t*>(p);
    const int bytes = n * (int)sizeof(E);
    int at = 0;
    const auto add = [&](uint64_t piece, int size) {
      piece <<= 8 * (at & 7);
      part[0] |= at < 8 ? piece : 0;
      part[1] |= at < 8 ? 0 : piece;
      at += size;
    };
    if (bytes & 8) { uint64_t x; __builtin_memcpy(&x, b, 8); add(x, 8); }
    if (bytes & 4) { uint32_t x; __builtin_memcpy(&x, b + at, 4); add(x, 4); }
    if (bytes & 2) { uint16_t x; __builtin_memcpy(&x, b + at, 2); add(x, 2); }
    if (sizeof(E) == 1 && (bytes & 1)) add(b[at], 1);
    __builtin_memcpy(&v, part, 16);
  }
  return v;
}

// Operands as in gsq_tile.hpp by way of registers, from any address: fetch() reads a wavefront's part of slab k,
// commit() writes it, or piece j of it, to LDS.
template <class E, int ROWS, int LOADS_ = ROWS / 8>
struct LooseAlong {
  static constexpr int LOADS = LOADS_, PER = 16 / (int)sizeof(E);
  const E* base;
  int64_t ld;
  int rows, ks, row0;
  i32x4 held[LOADS];

  __device__ __forceinline__ LooseAlong(const E* first, int64_t ld_, int rows_, int ks_, int wave)
      : base(first), ld(ld_), rows(rows_), ks(ks_), row0(wave * LOADS * 8) {}
  // The addresses are reckoned anew each time: with a uniform base and 32-bit lane offsets kept instead, 4096 rows
  // through 8190 x 4001 took 654 us, not 378.
  __device__ __forceinline__ void fetch(int k, uint8_t*) {
    const int lane = threadIdx.x & 63;
#pragma unroll
    for (int j = 0; j < LOADS; ++j) {
      const int row = row0 + j * 8 + (lane >> 3), at = (k * 8 + ((lane & 7) ^ swz(row))) * PER;
      held[j] = load_chunk(base + min(row, rows - 1) * ld + at, ks - at);
    }
  }
  __device__ __forceinline__ void commit(uint8_t* lds, int j) const {
    *reinterpret_cast<i32x4*>(lds + j * 1024 + (threadIdx.x & 63) * 16) = held[j];
  }
  __device__ __forceinline__ void commit(uint8_t* lds) const {
#pragma unroll
    for (int j = 0; j < LOADS; ++j) commit(lds, j);
  }
  static __device__ __forceinline__ i32x4 frag(const uint8_t* slab, int row0, int half, int lane) {
    return read_frag<i32x4>(slab, row0 + (lane & 15), half * 4 + (lane >> 4));
  }
};

template <class E, int COLS, int LOADS_ = COLS / 8>
struct LooseAcross {
  using Tight = SlabAcross<COLS, LOADS_>;
  static constexpr int LOADS = LOADS_;
  const uint8_t* base;
  uint32_t off[LOADS];       // bytes; below 64 x 2^22
  int64_t slab_bytes;
  int ks, wave;
  int left[LOADS];           // columns from the chunk's first

  __device__ __forceinline__ LooseAcross(const E* first, int64_t ld, int cols, int ks_, int wave_)
      : base(uniform(first)), slab_bytes(ld * (int64_t)sizeof(E) * kSlabRows), ks(ks_), wave(wave_) {
#pragma unroll
    for (int j = 0; j < LOADS; ++j) {
      int row, chunk;
      Tight::place((wave * LOADS + j) * 64 + (threadIdx.x & 63), row, chunk);
      off[j] = (uint32_t)row * (uint32_t)(ld * sizeof(E)) + (uint32_t)chunk * 16;
      left[j] = cols - chunk * 8;
    }
  }
  i32x4 held[LOADS];
  __device__ __forceinline__ void fetch(int k, uint8_t*) {
    const uint8_t* slab = base + k * slab_bytes;
#pragma unroll
    for (int j = 0; j < LOADS; ++j) {
      const int row = ((wave * LOADS + j) * 64 + (threadIdx.x & 63)) / Tight::PER_ROW;
      held[j] = load_chunk(reinterpret_cast<const E*>(slab + off[j]), k * kSlabRows + row < ks ? left[j] : 0);
    }
  }
  __device__ __forceinline__ void commit(uint8_t* lds, int j) const {
    *reinterpret_cast<i32x4*>(lds + j * 1024 + (threadIdx.x & 63) * 16) = held[j];
  }
  __device__ __forceinline__ void commit(uint8_t* lds) const {
#pragma unroll
    for (int j = 0; j < LOADS; ++j) commit(lds, j);
  }
  static __device__ __forceinline__ i32x4 frag(const uint8_t* slab, int col0, int half, int lane) {
    return Tight::frag(slab, col0, half, lane);
  }
};

// One of them in the ring of whole workgroups.
template <class Loose>
struct RingLoose : Loose {
  using Loose::Loose;
  static constexpr bool kCopied = false;
  __device__ __forceinline__ void prefetch(int k) { Loose::fetch(k, nullptr); }
  template <bool kEnd>
  __device__ __forceinline__ void load(int k, int j, uint8_t* lds) {
    Loose::commit(lds, j);
    if (j == Loose::LOADS - 1) prefetch(k + 1);
  }
};

// The same from aligned arrays, copied to LDS directly.
template <class Slab>
struct Copied : Slab {
  using Slab::Slab;
  __device__ __forceinline__ void fetch(int k, uint8_t* lds) {
#pragma unroll
    for (int j = 0; j < Slab::LOADS; ++j) Slab::template load<true>(k, j, lds);
  }
  __device__ __forceinline__ void commit(uint8_t*) const {}
};

// A wavefront's sums of a tile to LDS, rows of TN: a lane has row lane % 16 and four columns of a block.  The
// fours of a row are turned by the row, so that rows fall on different banks.
template <int TM, int TN, class Acc>
__device__ __forceinline__ void split_sums(const Acc (&acc)[TM / 16][TN / 16], uint8_t* own) {
  constexpr int FOURS = TN / 4;
  const int lane = threadIdx.x & 63;
#pragma unroll
  for (int i = 0; i < TM / 16; ++i)
#pragma unroll
    for (int j = 0; j < TN / 16; ++j) {
      const int row = i * 16 + (lane & 15), c = j * 4 + (lane >> 4);
      reinterpret_cast<Acc*>(own)[row * FOURS + (c ^ (row % FOURS))] = acc[i][j];
    }
}

// The c-th four of a row, added over the first `parts` wavefronts.
template <int TN, class Acc>
__device__ __forceinline__ Acc added_sums(const uint8_t* smem, int pitch, int parts, int row, int c) {
  constexpr int FOURS = TN / 4;
  Acc v = {};
  for (int w = 0; w < parts; ++w)
    v += reinterpret_cast<const Acc*>(smem + w * pitch)[row * FOURS + (c ^ (row % FOURS))];
  return v;
}

// Where the sums of a tile are added and stored: rows of TN in LDS, the first `parts` wavefronts' at `pitch`
// bytes from each other; with `mirror` also turned over.  Every thread of the workgroup calls it.
template <int TM, int TN, class Acc, class Columns>
__device__ __forceinline__ void store_added(uint8_t* smem, int pitch, int parts, Columns out, bool mirror, Columns turned) {
  constexpr int FOURS = TN / 4;
  __syncthreads();
  for (int f = threadIdx.x; f < TM * FOURS; f += blockDim.x) {
    const int row = f / FOURS, c = f % FOURS;
    out.begin(4 * c);
    const auto held = out.hold(row);
    const Acc v = added_sums<TN, Acc>(smem, pitch, parts, row, c);
    out.put(row, v, held);
    if (mirror) reinterpret_cast<Acc*>(smem)[row * FOURS + (c ^ (row % FOURS))] = v;
  }
  if (!mirror) return;
  __syncthreads();
  for (int f = threadIdx.x; f < TN * (TM / 4); f += blockDim.x) {
    const int row = 4 * (f % (TM / 4)), col = f / (TM / 4);
    Acc v;
#pragma unroll
    for (int r = 0; r < 4; ++r)
      v[r] = reinterpret_cast<const Acc*>(smem)[(row + r) * FOURS + ((col / 4) ^ ((row + r) % FOURS))][col % 4];
    turned.begin(row);
    turned.put(col, v, turned.hold(col));
  }
}

// A TM x TN tile: sums of slabs k = wave, wave + waves, ... < nk of each wavefront, added up, to `out`, and with
// `mirror` also turned over to `turned`.
// A wavefront reads a slab's fragments into registers, lets the next slab follow into the same LDS, and
// multiplies meanwhile.
template <class T, int TM, int TN, class A, class B, class Columns>
__device__ __forceinline__ void tile_split(A& a, B& b, int nk, uint8_t* smem, Columns out, bool mirror,
                                           Columns turned) {
  constexpr int MI = TM / 16, NJ = TN / 16;
  constexpr int A_SLAB = TM * ROW_BYTES, SLAB = A_SLAB + TN * ROW_BYTES;
  static_assert(TM * TN * 4 <= SLAB, "the sums take the slabs' place");
  const int lane = threadIdx.x & 63, waves = blockDim.x >> 6;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  uint8_t* const own = smem + wave * SLAB;
  typename T::acc acc[MI][NJ] = {};
  if (wave < nk) {
    a.fetch(wave, own);
    b.fetch(wave, own + A_SLAB);
    for (int k = wave; k < nk; k += waves) {
      a.commit(own);
      b.commit(own + A_SLAB);
      wait_all();
      typename T::frag fa[2][MI], fb[2][NJ];
#pragma unroll
      for (int h = 0; h < 2; ++h) {
#pragma unroll
        for (int i = 0; i < MI; ++i) fa[h][i] = __builtin_bit_cast(typename T::frag, A::frag(own, i * 16, h, lane));
#pragma unroll
        for (int j = 0; j < NJ; ++j) fb[h][j] = __builtin_bit_cast(typename T::frag, B::frag(own + A_SLAB, j * 16, h, lane));
      }
      wait_reads();
      if (k + waves < nk) {
        a.fetch(k + waves, own);
        b.fetch(k + waves, own + A_SLAB);
      }
#pragma unroll
      for (int h = 0; h < 2; ++h)
#pragma unroll
        for (int i = 0; i < MI; ++i)
#pragma unroll
          for (int j = 0; j < NJ; ++j) acc[i][j] = T::mfma(fb[h][j], fa[h][i], acc[i][j]);
    }
  }
  split_sums<TM, TN>(acc, own);
  store_added<TM, TN, typename T::acc>(smem, SLAB, min(waves, nk), out, mirror, turned);
}

}  // namespace
}  // namespace gsq
