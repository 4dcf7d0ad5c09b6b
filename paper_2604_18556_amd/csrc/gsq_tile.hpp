// The product of one output tile from two operands that move as slabs through a ring in LDS.
#pragma once
#include <hip/hip_runtime.h>
#include <stdint.h>

#include <atomic>
#include <type_traits>
#include <utility>

#include "gsq_plan.h"
#include "gsq_rows.hpp"
#include "gsq_slab.hpp"

namespace gsq {
namespace {

constexpr int kSlabRows = 64;        // rows of a slab that is read across k

// What lanes read where an operand has ended: zeros, in global memory so that it takes the same path.
__device__ const uint4 g_zeros[1] = {};
__device__ __forceinline__ const uint8_t* zeros() { return reinterpret_cast<const uint8_t*>(g_zeros); }

// A workgroup's tile: TM x TN outputs by four wavefronts (a quarter each), and slabs loaded AHEAD ahead of
// the one in use.  LDS holds a ring of AHEAD + 1 slabs of A and AHEAD of B.
template <int TM_, int TN_, int AHEAD_>
struct TileShape {
  static constexpr int TM = TM_, TN = TN_, AHEAD = AHEAD_;
  static constexpr int A_STAGES = AHEAD + 1, B_STAGES = AHEAD;
  static constexpr int A_SLAB = TM * ROW_BYTES, B_SLAB = TN * ROW_BYTES;
  static constexpr int B_BASE = A_STAGES * A_SLAB;
  static constexpr int A_LOADS = TM / 32, B_LOADS = TN / 32;   // 1 KB loads per wavefront and slab
  static constexpr int MI = TM / 32, NJ = TN / 32;             // 16 x 16 blocks per wavefront
  static constexpr size_t LDS = B_BASE + B_STAGES * B_SLAB;
  static_assert(LDS <= LDS_BYTES, "the ring fits the LDS");
};

// One block's product: B's columns are the instruction's rows, so that a lane's four results are four
// consecutive columns of a row.  The instruction is written out because the builtin gives its result other
// registers than its accumulator input once there are 64 of these, and moves them around.  The compiler
// then does not see when an accumulator can be read: acc_settled() waits for it.  The operands come from
// LDS reads, whose waits the compiler sets; no vector instruction writes them.  Both are checked in the built
// object code (tests/test_object_code.py).
template <class T>
__device__ __forceinline__ void mfma_block(typename T::acc& acc, const i32x4& b, const i32x4& a) {
  if constexpr (T::kDtype == GSQ_DT_BF16)
    asm volatile("v_mfma_f32_16x16x32_bf16 %0, %1, %2, %0" : "+a"(acc) : "v"(b), "v"(a));
  else if constexpr (T::kDtype == GSQ_DT_FP16)
    asm volatile("v_mfma_f32_16x16x32_f16 %0, %1, %2, %0" : "+a"(acc) : "v"(b), "v"(a));
  else
    asm volatile("v_mfma_i32_16x16x64_i8 %0, %1, %2, %0" : "+a"(acc) : "v"(b), "v"(a));
}

// Global->LDS copies of 16 bytes per lane, to `lds` + 16 lane.  Written out, so that the compiler does not
// make every transposing LDS read wait for all of them: the loop's own wait_vm() and barrier order them, and
// they return nothing to a register.  Addresses: a uniform base with 32-bit lane offsets, or one per lane.
// M0 holds the LDS address; nothing else in these kernels uses it (it is no register that the compiler keeps
// values in, nor one that it lets an asm declare).  A uniform base has to come from scalar instructions, as a
// slab's does that is reckoned from the operand's: one that a vector instruction wrote needs five instructions
// between, which the compiler does not see to here.  Both are checked in the built object code, too.
__device__ __forceinline__ uint32_t lds_address(const uint8_t* lds) {
  return (uint32_t)(uintptr_t)(const __attribute__((address_space(3))) uint8_t*)lds;
}
__device__ __forceinline__ void copy_to_lds(const uint8_t* base, uint32_t off, const uint8_t* lds) {
  asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %1, %2"
               :
               : "s"(__builtin_amdgcn_readfirstlane(lds_address(lds))), "v"(off), "s"(base)
               : "memory");
}
__device__ __forceinline__ void copy_to_lds(const uint8_t* src, const uint8_t* lds) {
  asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %1, off"
               :
               : "s"(__builtin_amdgcn_readfirstlane(lds_address(lds))), "v"(src)
               : "memory");
}

// An address that is the same in all lanes, in scalar registers.
__device__ __forceinline__ const uint8_t* uniform(const void* p) {
  const uint64_t v = reinterpret_cast<uint64_t>(p);
  const uint32_t lo = __builtin_amdgcn_readfirstlane((uint32_t)v), hi = __builtin_amdgcn_readfirstlane((uint32_t)(v >> 32));
  return reinterpret_cast<const uint8_t*>((uint64_t)hi << 32 | lo);
}

// An operand whose rows (of the output's side) run along k: a slab is 128 bytes of each of its rows, row r
// at r ROW_BYTES, chunks swizzled as swz() says.  Rows beyond the last one are read as the last one (their
// outputs are not stored), chunks beyond the end of k as zeros.
// kTracked: by the compiler's own copies, for kernels that have other loads in flight, which it can then
// wait for without waiting for these.
// LOADS_: copies of 1 KB that each of the wavefronts makes (ROWS / 8 in all).
template <int ROWS, int LOADS_ = ROWS / 32, bool kTracked = false>
struct SlabAlong {
  static constexpr bool kCopied = true;
  static constexpr int LOADS = LOADS_;
  const uint8_t* base;       // the tile's first row
  uint32_t off[LOADS];       // bytes; below 256 x 2^22
  int bytes;                 // of a row
  int chunk[LOADS];

  __device__ __forceinline__ SlabAlong(const void* first, int64_t row_bytes, int rows, int wave, int lane)
      : base(uniform(first)), bytes((int)row_bytes) {
#pragma unroll
    for (int j = 0; j < LOADS; ++j) {
      const int row = wave * (LOADS * 8) + j * 8 + (lane >> 3);
      chunk[j] = ((lane & 7) ^ swz(row)) * 16;
      off[j] = (uint32_t)min(row, rows - 1) * (uint32_t)row_bytes + chunk[j];
    }
  }
  template <bool kEnd>
  __device__ __forceinline__ void load(int k, int j, uint8_t* lds) const {
    const uint8_t* slab = base + (int64_t)k * ROW_BYTES;
    if constexpr (kTracked)
      load_rows(reinterpret_cast<const uint16_t*>(!kEnd || (int64_t)k * ROW_BYTES + chunk[j] < bytes ? slab + off[j]
                                                                                                   : zeros()),
                lds + j * 8 * ROW_BYTES);
    else if constexpr (kEnd)
      copy_to_lds((int64_t)k * ROW_BYTES + chunk[j] < bytes ? slab + off[j] : zeros(), lds + j * 8 * ROW_BYTES);
    else
      copy_to_lds(slab, off[j], lds + j * 8 * ROW_BYTES);
  }
  // 16 rows from `row0`, k of half a slab
  static __device__ __forceinline__ i32x4 frag(const uint8_t* slab, int row0, int half, int lane) {
    return read_frag<i32x4>(slab, row0 + (lane & 15), half * 4 + (lane >> 4));
  }
};

// An operand whose rows are k (16-bit elements, the output's side is contiguous): a slab is 64 rows of COLS
// elements.  The reads transpose: 16 lanes take four rows of 16 columns (32 bytes each) and each gets the
// four k of one column.  32 lanes read rows r .. r + 3 and r + 8 .. r + 11 at once: the 32-byte granules of
// a row are stored at granule ^ turn(row), so that those eight rows fall on distinct banks (narrow slabs have
// several rows in the 256 bytes of the banks, and less to turn).
// Rows beyond the end of k are read as zeros, columns beyond the last 16 bytes as those.
template <int COLS, int LOADS_ = COLS / 32>
struct SlabAcross {
  static constexpr bool kCopied = true;
  static constexpr int LOADS = LOADS_;
  static constexpr int PITCH = COLS * 2, PER_ROW = COLS / 8;   // bytes; 16-byte chunks
  const uint8_t* base;       // row 0 of k, the tile's first column
  uint32_t off[LOADS];       // bytes; below 64 x 2^22
  int64_t slab_bytes;        // from one slab to the next
  int rows;                  // of k
  int row[LOADS];

  static __device__ __forceinline__ int turn(int r) {
    return PITCH >= 256  ? (r & 3) | ((r >> 1) & 4)
           : PITCH == 128 ? ((r >> 1) & 1) | ((r >> 2) & 2)
           : PITCH == 64  ? (r >> 3) & 1
                          : 0;
  }
  // Row and chunk that are kept at the at-th 16 bytes of a slab.
  static __device__ __forceinline__ void place(int at, int& row, int& chunk) {
    const int c = at % PER_ROW;
    row = at / PER_ROW;
    chunk = ((c >> 1) ^ turn(row)) * 2 + (c & 1);
  }

  __device__ __forceinline__ SlabAcross(const void* first, int64_t row_bytes, int cols, int rows_, int wave,
                                        int lane)
      : base(uniform(first)), slab_bytes(row_bytes * kSlabRows), rows(rows_) {
#pragma unroll
    for (int j = 0; j < LOADS; ++j) {
      int chunk;
      place((wave * LOADS + j) * 64 + lane, row[j], chunk);
      off[j] = (uint32_t)row[j] * (uint32_t)row_bytes + (uint32_t)min(chunk * 16, cols * 2 - 16);
    }
  }
  template <bool kEnd>
  __device__ __forceinline__ void load(int k, int j, uint8_t* lds) const {
    const uint8_t* slab = base + k * slab_bytes;
    if constexpr (kEnd)
      copy_to_lds(k * kSlabRows + row[j] < rows ? slab + off[j] : zeros(), lds + j * 1024);
    else
      copy_to_lds(slab, off[j], lds + j * 1024);
  }
  static __device__ __forceinline__ i32x4 frag(const uint8_t* slab, int col0, int half, int lane) {
    typedef short s16x4 __attribute__((ext_vector_type(4)));
    typedef __attribute__((address_space(3))) s16x4* lds_ptr;
    const int r = half * 32 + (lane >> 4) * 8 + ((lane & 15) >> 2);
    const uint8_t* at = slab + r * PITCH + (((col0 >> 4) ^ turn(r)) << 5) + (lane & 3) * 8;
    union { s16x4 s[2]; i32x4 v; } u;
    u.s[0] = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_ptr)at);
    // bit 2 of a row does not enter its turn
    u.s[1] = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_ptr)(at + 4 * PITCH));
    return u.v;
  }
};

// f(0) .. f(N - 1) with the numbers as constants: loops whose bodies the compiler finds too long to unroll.
template <class F, int... I>
__device__ __forceinline__ void static_for_each(F& f, std::integer_sequence<int, I...>) {
  (f(std::integral_constant<int, I>{}), ...);
}
template <int N, class F>
__device__ __forceinline__ void static_for(F f) {
  static_for_each(f, std::make_integer_sequence<int, N>{});
}

// The tile: slabs 0 .. nk - 1, of which the last may end early (those past nk, for short sums, are zeros).
// 64 of k (128 of 8-bit integers) at a time move by direct global->LDS loads into the two rings.  A's extra
// buffer lets its slab k + AHEAD be loaded during the first half of slab k, B's during the second.  Fragment
// reads of the next half and slab loads are issued between the products, a load after every two reads.
// Blocks are walked back and forth: one operand of each product is the last one's.
//
// An operand need not be copied (!kCopied): its load(k, j, place) then writes 1 KB of slab k at that place (in
// SlabPacked's case relative to the wavefront's part), from what its prefetch() and the calls for slab k - 1 have
// fetched into registers.
template <class T, class S, class A, class B>
__device__ __forceinline__ void tile_ring(A& a, B& b, int nk,
                                          typename T::acc (&acc)[S::MI][S::NJ], uint8_t* smem) {
  const int tid = threadIdx.x, lane = tid & 63;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int wm = wave >> 1, wn = wave & 1;
#pragma unroll
  for (int i = 0; i < S::MI; ++i)
#pragma unroll
    for (int j = 0; j < S::NJ; ++j) acc[i][j] = typename T::acc{};
  acc_settled(acc);

  uint8_t* const a_wave = smem + wave * (S::A_SLAB / 4);
  uint8_t* const b_wave = smem + S::B_BASE + wave * (S::B_SLAB / 4);
  const int row_a = wm * (S::TM / 2), row_b = wn * (S::TN / 2);

  constexpr int kMfma = S::MI * S::NJ, kReads = S::MI + S::NJ;
  constexpr int kLess = S::MI < S::NJ ? S::MI : S::NJ;
  const auto read = [&](i32x4 (&fa)[S::MI], i32x4 (&fb)[S::NJ], int k, int half, int n) {
    // one of each in turn, then the rest of the longer side
    const bool of_b = n < 2 * kLess ? n % 2 == 1 : S::NJ > S::MI;
    const int i = n < 2 * kLess ? n / 2 : n - kLess;
    if (of_b)
      fb[i] = B::frag(smem + S::B_BASE + (k % S::B_STAGES) * S::B_SLAB, row_b + i * 16, half, lane);
    else
      fa[i] = A::frag(smem + (k % S::A_STAGES) * S::A_SLAB, row_a + i * 16, half, lane);
  };
  const auto half_slab = [&](const i32x4 (&fa)[S::MI], const i32x4 (&fb)[S::NJ], int n_reads, int n_loads,
                             auto&& next_read, auto&& next_load) {
    constexpr int kLoads = S::A_LOADS > S::B_LOADS ? S::A_LOADS : S::B_LOADS;
    constexpr int kOps = kReads + kReads / 2 > 3 * kLoads ? kReads + kReads / 2 : 3 * kLoads;
    constexpr int kStep = kMfma / kOps > 0 ? kMfma / kOps : 1;
    const auto op = [&](int o) {
      if (o % 3 == 2) { if (o / 3 < n_loads) next_load(o / 3); }
      else if (o - o / 3 < n_reads) next_read(o - o / 3);
    };
    static_for<kMfma>([&](auto at) {
      constexpr int n = decltype(at)::value;
      constexpr int i = n / S::NJ, j = i % 2 ? S::NJ - 1 - n % S::NJ : n % S::NJ;
      mfma_block<T>(acc[i][j], fb[j], fa[i]);
      if constexpr (n % kStep == 0) op(n / kStep);
    });
    constexpr int kDone = (kMfma + kStep - 1) / kStep;
    static_for<(kOps > kDone ? kOps - kDone : 0)>([&](auto at) { op(kDone + decltype(at)::value); });
  };
  const auto none = [](int) {};

  // p: first half of the current slab; q: second half
  i32x4 pa[S::MI], pb[S::NJ], qa[S::MI], qb[S::NJ];
  if constexpr (!A::kCopied) a.prefetch(0);
  if constexpr (!B::kCopied) b.prefetch(0);
#pragma unroll
  for (int k = 0; k < S::AHEAD; ++k) {
#pragma unroll
    for (int j = 0; j < S::A_LOADS; ++j) a.template load<true>(k, j, a_wave + k * S::A_SLAB);
#pragma unroll
    for (int j = 0; j < S::B_LOADS; ++j) b.template load<true>(k, j, b_wave + k * S::B_SLAB);
  }
  // copies of a slab; what is fetched besides makes the waits longer than need be, never shorter
  constexpr int kACopies = A::kCopied ? S::A_LOADS : 0, kSlabLoads = kACopies + (B::kCopied ? S::B_LOADS : 0);
  if constexpr (kSlabLoads > 0) wait_vm<(S::AHEAD - 1) * kSlabLoads>();
  slab_barrier();
#pragma unroll
  for (int n = 0; n < kReads; ++n) read(pa, pb, 0, 0, n);
  nk = max(nk, S::AHEAD);
  // one slab while AHEAD more are on their way; `end`: the one loaded may end early
  const auto step = [&](int kt, auto end) {
    constexpr bool kEnd = decltype(end)::value;
    half_slab(pa, pb, kReads, S::A_LOADS, [&](int n) { read(qa, qb, kt, 1, n); },
              [&](int j) {
                a.template load<kEnd>(kt + S::AHEAD, j, a_wave + ((kt + S::AHEAD) % S::A_STAGES) * S::A_SLAB);
              });
    __builtin_amdgcn_sched_barrier(0);   // every product of this half is issued before the wait
    // slab kt + 1 has landed (later ones, of kt + AHEAD only A's, may be in flight), and every
    // wavefront has read slab kt
    if constexpr (kSlabLoads > 0) wait_vm<(S::AHEAD - 2) * kSlabLoads + kACopies>();
    slab_barrier();
    half_slab(qa, qb, kReads, S::B_LOADS, [&](int n) { read(pa, pb, kt + 1, 0, n); },
              [&](int j) {
                b.template load<kEnd>(kt + S::AHEAD, j, b_wave + ((kt + S::AHEAD) % S::B_STAGES) * S::B_SLAB);
              });
    __builtin_amdgcn_sched_barrier(0);
  };
  int kt = 0;
  for (; kt < nk - S::AHEAD - 1; ++kt) step(kt, std::false_type{});
  if (kt < nk - S::AHEAD) step(kt++, std::true_type{});
  // the last slabs: nothing more to load
  for (; kt < nk - 1; ++kt) {
    half_slab(pa, pb, kReads, 0, [&](int n) { read(qa, qb, kt, 1, n); }, none);
    if constexpr (kSlabLoads > 0) wait_vm<0>();
    slab_barrier();
    half_slab(qa, qb, kReads, 0, [&](int n) { read(pa, pb, kt + 1, 0, n); }, none);
  }
  half_slab(pa, pb, kReads, 0, [&](int n) { read(qa, qb, nk - 1, 1, n); }, none);
  half_slab(qa, qb, 0, 0, none, none);
  acc_settled(acc);
}

// Place of the c-th four of row m of half a tile's results in LDS (fours): the fours of a row are turned, so that
// 16 rows, and every fourth of 64, fall on different banks.
template <class S>
__device__ __forceinline__ int result_place(int m, int c) {
  return m * (S::TN / 8) + (c ^ ((m ^ (m >> 2)) & 15));
}

// Where a thread stores results: four consecutive columns of one row after another, those in bounds (`rows`,
// `left` columns), rounded once to the nearest, ties to even; `four`: together, as they are whole and aligned.
// 8-bit integers' sums, exact in 32 bits, are scaled here.  begin(n) comes before any put().
template <class Out>
struct ResultColumns {
  Out* out;                // the tile's first element
  int64_t ld;
  int rows, cols;          // of the tile that exist
  bool four;
  bool add = false;        // to what is there (fp32)
  const float* row_scales = nullptr;
  const float* col_scales = nullptr;

  struct Held { f32x4 old; float scale; };   // what a put() needs from memory, asked for before
  Out* at = nullptr;
  int left = 0;
  f32x4 by = {1.f, 1.f, 1.f, 1.f};

  __device__ __forceinline__ void begin(int n) {
    at = out + n;
    left = cols - n;
    if (col_scales && left > 0)
#pragma unroll
      for (int c = 0; c < 4; ++c) by[c] = col_scales[n + min(c, left - 1)];
  }
  __device__ __forceinline__ Held hold(int m) const {
    Held h = {{0.f, 0.f, 0.f, 0.f}, 1.f};
    if (m < rows && left > 0) {
      if (row_scales) h.scale = row_scales[m];
      if (std::is_same<Out, float>::value && add)
#pragma unroll
        for (int c = 0; c < 4; ++c) h.old[c] = c < left ? (float)at[m * ld + c] : 0.f;
    }
    return h;
  }
  template <class Acc>
  __device__ __forceinline__ void put(int m, Acc sums, const Held& h) const {
    if (m >= rows || left <= 0) return;
    f32x4 v;
#pragma unroll
    for (int c = 0; c < 4; ++c) v[c] = (float)sums[c];
    if (row_scales)
#pragma unroll
      for (int c = 0; c < 4; ++c) v[c] = v[c] * h.scale * by[c];
    if (std::is_same<Out, float>::value && add) v += h.old;
    Out* const to = at + m * ld;
    if (four) {
      typedef Out o4 __attribute__((ext_vector_type(4)));
      *reinterpret_cast<o4*>(to) = __builtin_convertvector(v, o4);
    } else {
#pragma unroll
      for (int c = 0; c < 4; ++c)
        if (c < left) to[c] = (Out)v[c];
    }
  }
};

// The tile's results, half of its columns after the other through LDS (free of slabs by then), to `out`, whose
// lanes then follow each other along a row; with `mirror`, also turned over to `turned`.  Stores straight from
// the accumulators write pieces of 64 bytes, and their code, as long as there are accumulators and run through
// once, is fetched more slowly than it runs.  Eight rows are read from LDS before they are stored: one at a time
// took 350 clocks each.
template <class S, class Acc, class Columns>
__device__ __forceinline__ void tile_results(const Acc (&acc)[S::MI][S::NJ], uint8_t* smem, Columns out, bool mirror,
                                             Columns turned) {
  constexpr int FOURS = S::TN / 8, STEP = 256 / FOURS, kTimes = S::TM / STEP, kAtOnce = 8;
  static_assert(S::TM * FOURS * 16 <= (int)LDS_BYTES && FOURS % 16 == 0 && kTimes % kAtOnce == 0, "half a tile in LDS");
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  Acc* const part = reinterpret_cast<Acc*>(smem);
#pragma unroll 1
  for (int h = 0; h < 2; ++h) {
    __syncthreads();
    if ((wave & 1) == h)
#pragma unroll
      for (int i = 0; i < S::MI; ++i)
#pragma unroll
        for (int j = 0; j < S::NJ; ++j)
          part[result_place<S>((wave >> 1) * (S::TM / 2) + i * 16 + (lane & 15), j * 4 + (lane >> 4))] = acc[i][j];
    const int c = tid % FOURS;
    out.begin(h * (S::TN / 2) + 4 * c);
    __syncthreads();
#pragma unroll 1
    for (int m = tid / FOURS; m < S::TM; m += kAtOnce * STEP) {
      Acc v[kAtOnce];
      typename Columns::Held held[kAtOnce];
#pragma unroll
      for (int u = 0; u < kAtOnce; ++u) v[u] = part[result_place<S>(m + u * STEP, c)];
#pragma unroll
      for (int u = 0; u < kAtOnce; ++u) held[u] = out.hold(m + u * STEP);
#pragma unroll
      for (int u = 0; u < kAtOnce; ++u) out.put(m + u * STEP, v[u], held[u]);
    }
    if (mirror) {   // blocks of 4 x 4, neighbours along a transposed row
      const int m = tid % (S::TM / 4) * 4;
      turned.begin(m);
#pragma unroll 1
      for (int b = tid / (S::TM / 4); b < FOURS; b += 2 * (1024 / S::TM)) {
        Acc v[2][4];
        typename Columns::Held held[2][4];
#pragma unroll
        for (int u = 0; u < 2; ++u)
#pragma unroll
          for (int r = 0; r < 4; ++r) v[u][r] = part[result_place<S>(m + r, b + u * (1024 / S::TM))];
#pragma unroll
        for (int u = 0; u < 2; ++u)
#pragma unroll
          for (int n = 0; n < 4; ++n) held[u][n] = turned.hold(h * (S::TN / 2) + 4 * (b + u * (1024 / S::TM)) + n);
#pragma unroll
        for (int u = 0; u < 2; ++u)
#pragma unroll
          for (int n = 0; n < 4; ++n)
            turned.put(h * (S::TN / 2) + 4 * (b + u * (1024 / S::TM)) + n, Acc{v[u][0][n], v[u][1][n], v[u][2][n], v[u][3][n]},
                       held[u][n]);
      }
    }
  }
}

// The whole tile uses all the LDS; panels with fewer rows take lower ones, whose slabs last less long and
// are loaded further ahead.
using Whole = TileShape<256, 256, 2>;
using Half = TileShape<128, 256, 3>;
using Low = TileShape<64, 256, 3>;
// Two of these share a CU: one's loads and stores pass while the other multiplies.
using Quarter = TileShape<128, 128, 2>;

// The tile of y or dx that this workgroup has: up to `height` rows of one group, `width` columns.
struct RowsTile {
  int group;
  int64_t first;     // its first row
  int ms, n0;        // its rows, its first column
};

// Which one: the tiles of a group follow each other, and are spread over the XCDs so that each has a
// contiguous part of the group's tile order.  False: there are fewer.
__device__ __forceinline__ bool find_rows_tile(const GroupRows& rows, int height, int width, int cols, RowsTile& t) {
  const int tiles_n = (cols + width - 1) / width;
  PanelPlace at;
  if (!find_panel(rows, height, blockIdx.x / (unsigned)tiles_n, at)) return false;
  int tm, tn;
  tile_at(lin_of((int)(blockIdx.x - at.before * tiles_n), at.panels * tiles_n), at.panels, tiles_n, tm, tn);
  t.group = at.group;
  t.first = at.first + (int64_t)tm * height;
  t.ms = (int)min(at.end - t.first, (int64_t)height);
  t.n0 = tn * width;
  return true;
}

// A kernel that uses more LDS than the default limit needs leave for it, once on each device.
template <auto kKernel, class... Args>
hipError_t launch_lds(int64_t blocks, int threads, size_t lds, hipStream_t s, const Args&... args) {
  if (!fits_launch(blocks, threads)) return hipErrorInvalidConfiguration;
  if (lds > 64 * 1024) {
    static std::atomic<uint64_t> leave{0};   // a bit per device
    int dev = 0;
    hipError_t e = hipGetDevice(&dev);
    if (e != hipSuccess) return e;
    const uint64_t bit = dev < 64 ? (uint64_t)1 << dev : 0;
    if (!(leave.load(std::memory_order_relaxed) & bit)) {
      e = hipFuncSetAttribute(reinterpret_cast<const void*>(kKernel), hipFuncAttributeMaxDynamicSharedMemorySize,
                              (int)LDS_BYTES);
      if (e != hipSuccess) return e;
      leave.fetch_or(bit, std::memory_order_relaxed);
    }
  }
  kKernel<<<(unsigned)blocks, threads, lds, s>>>(args...);
  return hipGetLastError();
}
template <auto kKernel, class... Args>
hipError_t launch_ring(int64_t blocks, hipStream_t s, const Args&... args) {
  return launch_lds<kKernel>(blocks, 256, LDS_BYTES, s, args...);
}

bool aligned16(const void* p) { return (reinterpret_cast<uintptr_t>(p) & 15) == 0; }

// Results can be stored four at a time: whole rows of them, at aligned addresses.
bool four_at_once(const void* out, int32_t dtype, int32_t cols) {
  const uintptr_t bytes = dtype == GSQ_DT_FP32 ? 16 : 8;
  return cols % 4 == 0 && (reinterpret_cast<uintptr_t>(out) & (bytes - 1)) == 0;
}

}  // namespace
}  // namespace gsq
