// Low-rank adapters of many requests: y = base + s B (A x) and its gradients, the adapter being that of the row's
// segment.
//
// A product through a low rank is two products whose inner results are small: hidden goes to memory in fp32 (the gradients
// need it again), and both kernels of a call are bound by reading x and by reading and writing y, not by the matrix cores
// (busy 0.03 and 0.09 of the time at 4096 rows, 4096 -> 64 -> 14336: 20 us for A x, 58 us for y).
#include <hip/hip_runtime.h>

#include <algorithm>

#include "gsq_adapter.h"
#include "gsq_split.hpp"
#include "gsq_walk.h"

namespace gsq {
namespace {

// The adapter of a segment, or -1.
__device__ __forceinline__ int adapter_of(const AdapterArgs& p, int segment) {
  const int e = p.index ? p.index[segment] : segment;
  return (unsigned)e < (unsigned)p.adapters ? e : -1;
}
__device__ __forceinline__ float scale_of(const AdapterArgs& p, int e) { return p.scales ? p.scales[e] : 1.f; }

// ------------------------------------------------------------------ hidden = A x, dhidden = s B^T dy
// Where the sums of a tile are stored: times the adapter's scale, in fp32.
struct HiddenColumns {
  float* out;
  int ld, rows, cols;
  bool four;
  float scale;
  struct Held {};
  int at = 0;
  __device__ __forceinline__ void begin(int n) { at = n; }
  __device__ __forceinline__ Held hold(int) const { return {}; }
  __device__ __forceinline__ void put(int m, f32x4 v, Held) const {
    if (m >= rows || at >= cols) return;
    v *= scale;
    float* to = out + (int64_t)m * ld + at;
    if (four) {
      *reinterpret_cast<f32x4*>(to) = v;
    } else {
#pragma unroll
      for (int c = 0; c < 4; ++c)
        if (at + c < cols) to[c] = v[c];
    }
  }
};

// A tile of TM rows x TN of the rank, by wavefronts that share the sum.  4096 rows of 4096 at rank 64 take 20 us (12 with
// warm caches): 16 rows to a workgroup read the whole of A each, 0.17 GB through the L2s for 0.03 of x, and wait 0.6 of
// the time.  Non-temporal copies of x, slabs in another order for each workgroup, and neighbouring slabs to a wavefront
// changed nothing.
template <class T, int kForm, int TM, int TN, bool kLoose>
__device__ __forceinline__ void down_tile(const AdapterArgs& p, int e, int64_t first, int ms, int n0, uint8_t* smem) {
  using E = typename T::elem;
  const int lane = threadIdx.x & 63, ks = kForm == kForward ? p.I : p.O;
  const HiddenColumns out{p.hidden + first * p.q + n0, p.q, ms, p.q - n0, p.vector_hidden != 0,
                          kForm == kForward || e < 0 ? 1.f : scale_of(p, e)};
  if (e < 0) {
    for (int f = threadIdx.x; f < ms * TN; f += blockDim.x)
      if (n0 + f % TN < p.q) out.out[(int64_t)(f / TN) * p.q + f % TN] = 0.f;
    return;
  }
  const int nk = (ks + kSlabRows - 1) / kSlabRows;
  const E* in = static_cast<const E*>(kForm == kForward ? p.x : p.dy) + first * ks;
  const E* w = static_cast<const E*>(kForm == kForward ? p.a : p.b) + (int64_t)e * p.q * ks;
  if constexpr (kLoose) {
    LooseAlong<E, TM> a(in, ks, ms, ks, 0);
    if constexpr (kForm == kForward) {
      LooseAlong<E, TN> b(w + (int64_t)n0 * ks, ks, p.q - n0, ks, 0);
      tile_split<T, TM, TN>(a, b, nk, smem, out, false, out);
    } else {
      LooseAcross<E, TN> b(w + n0, p.q, p.q - n0, ks, 0);
      tile_split<T, TM, TN>(a, b, nk, smem, out, false, out);
    }
  } else {
    Copied<SlabAlong<TM, TM / 8>> a(in, (int64_t)ks * 2, ms, 0, lane);
    if constexpr (kForm == kForward) {
      Copied<SlabAlong<TN, TN / 8>> b(w + (int64_t)n0 * ks, (int64_t)ks * 2, p.q - n0, 0, lane);
      tile_split<T, TM, TN>(a, b, nk, smem, out, false, out);
    } else {
      Copied<SlabAcross<TN, TN / 8>> b(w + n0, (int64_t)p.q * 2, p.q - n0, ks, 0, lane);
      tile_split<T, TM, TN>(a, b, nk, smem, out, false, out);
    }
  }
}

// Wavefronts that share a tile: as many as the LDS holds slabs for, sixteen at most.
template <int TM, int TN>
constexpr int kDownWaves = (TM + TN) * ROW_BYTES * 16 < (int)LDS_BYTES ? 16 : 8;

template <class T, int kForm, int TM, int TN, bool kLoose>
__global__ __launch_bounds__((64 * kDownWaves<TM, TN>)) void k_adapter_down(AdapterArgs p) {
  extern __shared__ __attribute__((aligned(16))) uint8_t smem[];
  const int tiles_n = (p.q + TN - 1) / TN;
  PanelPlace at;
  if (!find_panel(p.rows, TM, blockIdx.x / (unsigned)tiles_n, at)) return;
  int tm, tn;
  tile_at(lin_of((int)(blockIdx.x - at.before * tiles_n), at.panels * tiles_n), at.panels, tiles_n, tm, tn);
  const int64_t first = at.first + (int64_t)tm * TM;
  const int ms = (int)min(at.end - first, (int64_t)TM);
  const int e = adapter_of(p, at.group);
  if (TM > 16 && ms <= 16)
    down_tile<T, kForm, 16, TN, kLoose>(p, e, first, ms, tn * TN, smem);
  else
    down_tile<T, kForm, TM, TN, kLoose>(p, e, first, ms, tn * TN, smem);
}

// ------------------------------------------------------------------ y = base + s B hidden, dx = base + A^T dhidden
// hidden is split into two 16-bit parts, so that the product keeps 16 bits of its mantissa (bf16; fp16 22) and runs at
// the matrix cores' 16-bit rate twice: by fp32 instructions it would take eight times as long.  fp16 rows are taken
// times a power of two that brings their largest value to 2^13 .. 2^14, as its exponent would not hold both parts.
//
// 64 columns of the adapter's matrix are the instructions' rows, in four blocks: row 4 g + c of block j is column
// up_column(g, j) + c, so that a lane's results are twice eight neighbouring columns of one row of y, and four lanes
// store 64 bytes of it together.
constexpr int kUpCols = 64, kUpWaves = 4, kUpRows = 16 * kUpWaves;
constexpr int kUpBlock = 32 * kUpCols * 2;     // bytes of 32 of the rank for these columns

__device__ __forceinline__ int up_column(int g, int j) { return 32 * (j >> 1) + 8 * g + 4 * (j & 1); }

// Eight hidden values of a row from k on, those from q on zeros.
__device__ __forceinline__ void load_hidden(const float* row, int k, int q, float (&v)[8]) {
  if (k + 8 <= q) {
    __builtin_memcpy(v, row + k, 32);
  } else {
#pragma unroll
    for (int i = 0; i < 8; ++i) v[i] = k + i < q ? row[k + i] : 0.f;
  }
}

// The power of two that a row is taken by: found by the four lanes that share the row.
template <class T>
__device__ __forceinline__ float hidden_power(const float* row, int q) {
  if constexpr (T::kDtype != GSQ_DT_FP16) return 1.f;
  float top = 0.f;
  for (int k = 8 * ((threadIdx.x & 63) >> 4); k < q; k += 32) {
    float v[8];
    load_hidden(row, k, q, v);
#pragma unroll
    for (int c = 0; c < 8; ++c) top = fmaxf(top, fabsf(v[c]));
  }
  top = fmaxf(top, __shfl_xor(top, 16, 64));
  top = fmaxf(top, __shfl_xor(top, 32, 64));
  // infinities pass as they are (and NaN, which fmaxf leaves out); what is very small, as far as it goes
  if (!(top > 0.f && top < __builtin_huge_valf())) return 1.f;
  return ldexpf(1.f, 13 - max((int)(__float_as_uint(top) >> 23) - 127, -100));
}

template <class T>
__device__ __forceinline__ void split_hidden(const float* row, int k, int q, float by, typename T::frag& hi,
                                             typename T::frag& lo) {
  using E = typename T::elem;
  // the largest of 16 bits: what is finite and would be rounded beyond it (bf16) has its rest in the second part, as have
  // infinities and NaN, whole
  constexpr float kTop = T::kDtype == GSQ_DT_FP16 ? 65504.f : 0x1.fep127f;
  float v[8];
  load_hidden(row, k + 8 * ((threadIdx.x & 63) >> 4), q, v);
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    const float x = v[i] * by;
    const E h = (E)__builtin_amdgcn_fmed3f(x, -kTop, kTop);
    hi[i] = h;
    lo[i] = (E)(x - (float)h);
  }
}

// 64 columns of the matrix in LDS, in blocks of 32 of the rank; 256 lanes fill a block together, 16 bytes each: at() says
// where the lane's 16 bytes of a block come from (16-byte aligned arrays; nullptr: zeros), held() what they hold else.
// B, whose rows run along the rank: a column has 64 bytes of a block, its four chunks turned so that fragment reads
// fall on distinct banks.
template <class T>
struct UpAlong {
  using E = typename T::elem;
  const E* w;                  // the adapter's
  int cols, q;
  static __device__ __forceinline__ int turn(int col) { return -(col >> 3) & 3; }
  __device__ __forceinline__ const E* place(int n0, int k, int t, int& left) const {
    const int col = t >> 2, at = k + 8 * ((t & 3) ^ turn(col));
    left = q - at;
    return w + (int64_t)min(n0 + col, cols - 1) * q + at;
  }
  static __device__ __forceinline__ typename T::frag frag(const uint8_t* block, int j) {
    const int lane = threadIdx.x & 63, i = lane & 15, col = up_column(i >> 2, j) + (i & 3);
    return *reinterpret_cast<const typename T::frag*>(block + col * 64 + (((lane >> 4) ^ turn(col)) << 4));
  }
};
// A, whose rows are the rank: 32 rows of 64 columns, read by transposing reads.
template <class T>
struct UpAcross {
  using E = typename T::elem;
  using Slab = SlabAcross<kUpCols>;
  const E* w;
  int cols, q;
  __device__ __forceinline__ const E* place(int n0, int k, int t, int& left) const {
    int row, chunk;
    Slab::place(t, row, chunk);
    const int col = n0 + chunk * 8;
    left = k + row < q ? cols - col : 0;
    return w + (int64_t)(k + row) * cols + col;
  }
  static __device__ __forceinline__ typename T::frag frag(const uint8_t* block, int j) {
    typedef short s16x4 __attribute__((ext_vector_type(4)));
    typedef __attribute__((address_space(3))) s16x4* lds_ptr;
    const int lane = threadIdx.x & 63, r = (lane >> 4) * 8 + ((lane & 15) >> 2);
    const int col = up_column(lane & 3, j);
    const uint8_t* at = block + r * Slab::PITCH + (((col >> 4) ^ Slab::turn(r)) << 5) + (col & 15) * 2;
    union { s16x4 s[2]; typename T::frag v; } u;
    u.s[0] = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_ptr)at);
    u.s[1] = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_ptr)(at + 4 * Slab::PITCH));
    return u.v;
  }
};

// One block of the matrix to LDS: copied directly (kCopied: 16-byte aligned), or by way of registers.
template <class W, bool kCopied>
struct UpBlock {
  i32x4 held;
  __device__ __forceinline__ void fetch(const W& w, int n0, int k, uint8_t* block) {
    int left;
    const int t = threadIdx.x % (64 * kUpWaves);
    const auto* from = w.place(n0, k, t, left);
    if constexpr (kCopied)
      copy_to_lds(left > 0 ? reinterpret_cast<const uint8_t*>(from) : zeros(), block + (t & ~63) * 16);
    else
      held = load_chunk(from, left);
  }
  __device__ __forceinline__ void commit(uint8_t* block) const {
    if constexpr (!kCopied) *reinterpret_cast<i32x4*>(block + (threadIdx.x % (64 * kUpWaves)) * 16) = held;
  }
};

// How y is gone through: value by value, by 16 bytes (rows are whole pieces), or by these past the caches.
enum { kNarrow = 0, kWide = 1, kStream = 2 };

// Of 16 rows of y, 64 columns: a lane has columns 8 g .. and 32 + 8 g .., eight each, of row m = lane % 16 (g = lane /
// 16).  In memory the lane goes to two half-rows of 64 bytes, those of rows m % 8 and m % 8 + 8, so that eight lanes
// have a row's whole 128 bytes at once; the lanes 8 apart exchange what is the other's.
template <class E, int kBy>
struct Sixteen {
  typedef E vec __attribute__((ext_vector_type(8)));
  i32x4 part[2];
  static __device__ __forceinline__ void exchange(i32x4& a, i32x4& b) {
    const bool high = threadIdx.x & 8;
    i32x4 mine = high ? a : b, other;
#pragma unroll
    for (int i = 0; i < 4; ++i) other[i] = __builtin_amdgcn_update_dpp(0, mine[i], 0x128, 0xf, 0xf, true);   // row_ror:8
    a = high ? other : a;
    b = high ? b : other;
  }
  // `first`: row 0's element at column 0; columns n .. below cols, rows below `rows` (none: zeros)
  __device__ __forceinline__ void load(const E* first, int64_t ld, int rows, int n, int cols) {
    const int lane = threadIdx.x & 63, m = lane & 15, g = lane >> 4;
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      if constexpr (kBy != kNarrow) {
        const int r = (m & 7) + 8 * h, c = n + 32 * (m >> 3) + 8 * g;
        const i32x4* from = reinterpret_cast<const i32x4*>(first + r * ld + c);
        part[h] = i32x4{};
        if (r < rows && c < cols) part[h] = kBy == kStream ? __builtin_nontemporal_load(from) : *from;
      } else {
        const int c = n + 32 * h + 8 * g;
        vec v;
#pragma unroll
        for (int i = 0; i < 8; ++i) v[i] = m < rows && c + i < cols ? first[m * ld + c + i] : (E)0.f;
        part[h] = __builtin_bit_cast(i32x4, v);
      }
    }
  }
  // sums times s and what was loaded, rounded once
  __device__ __forceinline__ void store(const f32x4 (&acc)[4], float s, E* first, int64_t ld, int rows, int n, int cols) const {
    const int lane = threadIdx.x & 63, m = lane & 15, g = lane >> 4;
    i32x4 old[2] = {part[0], part[1]}, res[2];
    if constexpr (kBy != kNarrow) exchange(old[0], old[1]);
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      const vec o = __builtin_bit_cast(vec, old[h]);
      vec r;
#pragma unroll
      for (int i = 0; i < 8; ++i) r[i] = (E)fmaf(acc[2 * h + i / 4][i % 4], s, (float)o[i]);
      res[h] = __builtin_bit_cast(i32x4, r);
    }
    if constexpr (kBy != kNarrow) exchange(res[0], res[1]);
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      if constexpr (kBy != kNarrow) {
        const int r = (m & 7) + 8 * h, c = n + 32 * (m >> 3) + 8 * g;
        i32x4* to = reinterpret_cast<i32x4*>(first + r * ld + c);
        if (r < rows && c < cols) {
          if constexpr (kBy == kStream)
            __builtin_nontemporal_store(res[h], to);
          else
            *to = res[h];
        }
      } else {
        const int c = n + 32 * h + 8 * g;
        const vec r = __builtin_bit_cast(vec, res[h]);
#pragma unroll
        for (int i = 0; i < 8; ++i)
          if (m < rows && c + i < cols) first[m * ld + c + i] = r[i];
      }
    }
  }
};

// Rows without an adapter: the base, or zeros, by pieces as y is gone through, four of a lane on their way at once (4096
// rows of 14336 53 us with the call's first kernel, 85 value by value).
template <class E, int kBy>
__device__ __forceinline__ void copy_base(const AdapterArgs& p, int64_t first, int ms, int n0, int cols, int ns) {
  using Piece = std::conditional_t<kBy == kNarrow, E, i32x4>;
  constexpr int PER = sizeof(Piece) / sizeof(E), AHEAD = 4;
  if (p.base == p.out) return;
  const E* const base = static_cast<const E*>(p.base) + first * ns + n0;
  E* const out = static_cast<E*>(p.out) + first * ns + n0;
  const int pieces = cols / PER, all = ms * pieces;
  for (int f0 = threadIdx.x; f0 < all; f0 += AHEAD * blockDim.x) {
    Piece v[AHEAD];
    int64_t at[AHEAD];
#pragma unroll
    for (int u = 0; u < AHEAD; ++u) {
      const int f = min(f0 + u * (int)blockDim.x, all - 1), r = f / pieces;
      at[u] = (int64_t)r * ns + (f - r * pieces) * PER;
      v[u] = Piece{};
      if (p.base) v[u] = kBy == kStream ? __builtin_nontemporal_load(reinterpret_cast<const Piece*>(base + at[u]))
                                        : *reinterpret_cast<const Piece*>(base + at[u]);
    }
#pragma unroll
    for (int u = 0; u < AHEAD; ++u) {
      if (f0 + u * (int)blockDim.x >= all) break;
      if constexpr (kBy == kStream)
        __builtin_nontemporal_store(v[u], reinterpret_cast<Piece*>(out + at[u]));
      else
        *reinterpret_cast<Piece*>(out + at[u]) = v[u];
    }
  }
}

// Waits until the blocks that this wavefront has copied are there, of whose later accesses `after` are at least on
// their way still.
__device__ __forceinline__ void wait_blocks(int after) {
  __atomic_signal_fence(__ATOMIC_SEQ_CST);
  if (after == 4)
    wait_vm<4>();
  else if (after == 2)
    wait_vm<2>();
  else
    wait_vm<0>();
  __atomic_signal_fence(__ATOMIC_SEQ_CST);
}

// Panels of 64 rows (16 to a wavefront) and `steps` times 64 columns.  A panel's hidden stays in registers as long as its
// rank fits KS blocks.  While a step is multiplied, the matrix of the next is on its way to LDS, and the base of the next
// two to registers; but before a step's base enters its sums everything that is on its way is waited for, as the built
// code cannot count on the younger loads, which stand under lane masks.  4096 rows of 14336 with a base at rank 64: 58 us,
// 235 MB of base and y at 4.1 TB/s (a copy of as much takes 45), waiting half of the time.  With cold caches 60, and 116
// with the matrix read by each wavefront for itself, 92 from LDS but 32 bytes of a row stored at a time, 80 with 64, 78
// with whole lines that the caches keep.  Twice the columns at a step, a panel's workgroups on neighbouring columns at
// each step, and each XCD on columns of its own changed nothing or cost a tenth.
template <class T, int kForm, int KS, bool kCopied, int kBy>
__global__ __launch_bounds__(64 * kUpWaves) void k_adapter_up(AdapterArgs p, int steps, int chunks) {
  using E = typename T::elem;
  using W = std::conditional_t<kForm == kForward, UpAlong<T>, UpAcross<T>>;
  __shared__ __attribute__((aligned(16))) uint8_t smem[2][KS * kUpBlock];
  const int ns = kForm == kForward ? p.O : p.I;
  PanelPlace at;
  if (!find_panel(p.rows, kUpRows, blockIdx.x / (unsigned)chunks, at)) return;
  const int64_t first = at.first + (blockIdx.x / (unsigned)chunks - at.before) * kUpRows;
  const int ms = (int)min(at.end - first, (int64_t)kUpRows), wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int n0 = (blockIdx.x % (unsigned)chunks) * steps * kUpCols, n1 = min(n0 + steps * kUpCols, ns);
  const int e = adapter_of(p, at.group);
  if (e < 0) return copy_base<E, kBy>(p, first, ms, n0, n1 - n0, ns);
  const W w{static_cast<const E*>(kForm == kForward ? p.b : p.a) + (int64_t)e * p.q * ns, ns, p.q};
  const float scale = kForm == kForward ? scale_of(p, e) : 1.f;

  const int rows = ms - 16 * wave;             // of this wavefront, if any
  const float* hid = p.hidden + (first + min(16 * wave + (int)(threadIdx.x & 15), ms - 1)) * p.q;
  const E* base = static_cast<const E*>(p.base) + (first + 16 * wave) * ns;
  E* out = static_cast<E*>(p.out) + (first + 16 * wave) * ns;
  const int base_rows = p.base ? rows : 0;
  const int passes = (p.q + 32 * KS - 1) / (32 * KS);

  UpBlock<W, kCopied> blocks[KS];
  Sixteen<E, kBy> even, odd;
  even.load(base, ns, base_rows, n0, n1);
  odd.load(base, ns, base_rows, n0 + kUpCols, n1);
#pragma unroll
  for (int s = 0; s < KS; ++s) blocks[s].fetch(w, n0, 32 * s, smem[0] + s * kUpBlock);
  const float by = hidden_power<T>(hid, p.q), undo = scale / by;     // by is a power of two
  typename T::frag hi[KS], lo[KS];
#pragma unroll
  for (int s = 0; s < KS; ++s) split_hidden<T>(hid, 32 * s, p.q, by, hi[s], lo[s]);
#pragma unroll
  for (int s = 0; s < KS; ++s) blocks[s].commit(smem[0] + s * kUpBlock);
  int parity = 0, after = 0;
  const auto step = [&](int n, Sixteen<E, kBy>& old) {
    f32x4 acc[4] = {};
    for (int pass = 0; pass < passes; ++pass) {
      uint8_t* const here = smem[parity];
      uint8_t* const there = smem[parity ^ 1];
      if constexpr (kCopied) wait_blocks(after);
      slab_barrier();
      const bool last = pass == passes - 1, more = !last || n + kUpCols < n1;
      if (more)
#pragma unroll
        for (int s = 0; s < KS; ++s)
          blocks[s].fetch(w, last ? n + kUpCols : n, (last ? 0 : pass + 1) * 32 * KS + 32 * s, there + s * kUpBlock);
      if (rows > 0) {
        if (passes > 1)
#pragma unroll
          for (int s = 0; s < KS; ++s) split_hidden<T>(hid, (pass * KS + s) * 32, p.q, by, hi[s], lo[s]);
#pragma unroll
        for (int s = 0; s < KS; ++s) {
          typename T::frag f[4];
#pragma unroll
          for (int j = 0; j < 4; ++j) f[j] = W::frag(here + s * kUpBlock, j);
#pragma unroll
          for (int j = 0; j < 4; ++j) acc[j] = T::mfma(f[j], hi[s], acc[j]);
#pragma unroll
          for (int j = 0; j < 4; ++j) acc[j] = T::mfma(f[j], lo[s], acc[j]);
        }
      }
      if (!kCopied && more)
#pragma unroll
        for (int s = 0; s < KS; ++s) blocks[s].commit(there + s * kUpBlock);
      parity ^= 1;
      after = 0;
    }
    if (rows <= 0) return;
    old.store(acc, undo, out, ns, rows, n, n1);
    const int ahead = n + 2 * kUpCols;
    if (ahead < n1) old.load(base, ns, base_rows, ahead, n1);
    // with more than eight rows two stores, and two loads unless the columns end within that step
    if (kBy != kNarrow && rows > 8) after = base_rows && ahead + kUpCols <= n1 ? 4 : 2;
  };
  for (int n = n0; n < n1; n += 2 * kUpCols) {
    step(n, even);
    if (n + kUpCols < n1) step(n + kUpCols, odd);
  }
}

// Segments of few rows: panels of 16 and 64 columns to a wavefront, straight from memory; no wavefront waits for another.
template <class T, int kForm, int kBy>
__global__ __launch_bounds__(64 * kUpWaves) void k_adapter_up_few(AdapterArgs p) {
  using E = typename T::elem;
  using W = std::conditional_t<kForm == kForward, UpAlong<T>, UpAcross<T>>;
  __shared__ __attribute__((aligned(16))) uint8_t smem[kForm == kForward ? 1 : kUpWaves][kUpBlock];
  const int ns = kForm == kForward ? p.O : p.I, wide = kUpCols * kUpWaves, tiles_n = (ns + wide - 1) / wide;
  PanelPlace at;
  if (!find_panel(p.rows, 16, blockIdx.x / (unsigned)tiles_n, at)) return;
  const int64_t first = at.first + (blockIdx.x / (unsigned)tiles_n - at.before) * 16;
  const int ms = (int)min(at.end - first, (int64_t)16), wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int e = adapter_of(p, at.group), n_all = (blockIdx.x % (unsigned)tiles_n) * wide;
  if (e < 0) return copy_base<E, kBy>(p, first, ms, n_all, min(ns - n_all, wide), ns);
  const int n0 = n_all + wave * kUpCols;
  if (n0 >= ns) return;
  const W w{static_cast<const E*>(kForm == kForward ? p.b : p.a) + (int64_t)e * p.q * ns, ns, p.q};
  const int lane = threadIdx.x & 63;
  const float* hid = p.hidden + (first + min(lane & 15, ms - 1)) * p.q;
  Sixteen<E, kBy> old;
  old.load(static_cast<const E*>(p.base) + first * ns, ns, p.base ? ms : 0, n0, ns);
  const float by = hidden_power<T>(hid, p.q);
  f32x4 acc[4] = {};
  for (int k = 0; k < p.q; k += 32) {
    typename T::frag f[4], hi, lo;
    if constexpr (kForm == kForward) {
      const int i = lane & 15, at_k = k + 8 * (lane >> 4);
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        const int c = min(n0 + up_column(i >> 2, j) + (i & 3), ns - 1);
        f[j] = __builtin_bit_cast(typename T::frag, load_chunk(w.w + (int64_t)c * p.q + at_k, p.q - at_k));
      }
    } else {
      uint8_t* const own = smem[wave];
      i32x4 v[4];
#pragma unroll
      for (int u = 0; u < 4; ++u) {
        int left;
        const E* from = w.place(n0, k, u * 64 + lane, left);
        v[u] = load_chunk(from, left);
      }
      wait_reads();                            // of the block before
#pragma unroll
      for (int u = 0; u < 4; ++u) *reinterpret_cast<i32x4*>(own + (u * 64 + lane) * 16) = v[u];
      wait_reads();
#pragma unroll
      for (int j = 0; j < 4; ++j) f[j] = W::frag(own, j);
    }
    split_hidden<T>(hid, k, p.q, by, hi, lo);
#pragma unroll
    for (int j = 0; j < 4; ++j) acc[j] = T::mfma(f[j], hi, acc[j]);
#pragma unroll
    for (int j = 0; j < 4; ++j) acc[j] = T::mfma(f[j], lo, acc[j]);
  }
  old.store(acc, (kForm == kForward ? scale_of(p, e) : 1.f) / by, static_cast<E*>(p.out) + first * ns, ns, ms, n0, ns);
}

// ------------------------------------------------------------------ dA, dB: sums over an adapter's rows
// The instructions' rows are the rank, their columns those of x (or dy), and both run across their arrays.  x comes to
// LDS in slabs of 32 rows, two of them for each wavefront, and is read by transposing reads; a lane reads its eight hidden
// values of a column itself.  Two slabs are asked for at first; later a slab is asked for while the one before is
// multiplied, and waited for right after, copies and all, as hidden goes to registers on several ways that meet.
// fp32 instructions would need no transposing, but take five times as long as the bf16 ones of the exact parts that
// hidden is split into, three of 8 bits (fp16 x: two parts, of whose products those below 2^-24 of the whole are left out).
// 4096 rows of 4096 + 14336 columns in four adapters of rank 32: 43 us, 0.15 GB at 3.5 TB/s (92 by fp32 instructions, with
// 64-row slabs one at a time 50); the largest adapter has half of the rows, and the rounds of workgroups end unevenly.
// One adapter has a workgroup for each 128 columns only: 8192 rows of 4096 + 4096 at rank 16 61 us.
constexpr int kWeightCols = 128, kWeightBlocks = kWeightCols / 16;
constexpr int kWeightRows = 32, kWeightSlab = kWeightRows * kWeightCols * 2;

// The slabs of an adapter's rows, of which each wavefront takes every waves-th.
struct AdapterSlabs {
  const AdapterArgs& p;
  int e, s0 = 0;
  uint64_t mine = 0;           // segments from s0 on that are left
  SlabWalk walk;

  __device__ __forceinline__ AdapterSlabs(const AdapterArgs& args, int adapter, int wave) : p(args), e(adapter), walk(wave) {
    if (!p.index) {
      if (e < p.rows.groups) enter(e);
    } else {
      look();
    }
  }
  __device__ __forceinline__ void enter(int segment) {
    int64_t first, end;
    group_rows(p.rows, segment, first, end);
    walk.enter(first, end);
  }
  __device__ __forceinline__ void look() {
    const int lane = threadIdx.x & 63, s = min(s0 + lane, p.rows.groups - 1);
    mine = __ballot(s0 + lane < p.rows.groups && p.index[s] == e);
  }
  // The next slab: its first row and how many it has.  Once there is none, there is none again.
  __device__ __forceinline__ bool next(int64_t& first, int& rows) {
    while (!walk.take(kWeightRows, blockDim.x >> 6, first, rows)) {
      if (!p.index) return false;
      while (!mine) {
        s0 += 64;
        if (s0 >= p.rows.groups) return false;
        look();
      }
      enter(s0 + __builtin_ctzll(mine));
      mine &= mine - 1;
    }
    return true;
  }
};

// Parts of 8 bits, cut off one after another, that add up to v exactly (24 bits in three; what is not finite makes the
// later ones NaN).
template <int N>
__device__ __forceinline__ void exact_parts(const float (&v)[8], bf16x8 (&part)[N]) {
  uint32_t rest[8];
#pragma unroll
  for (int i = 0; i < 8; ++i) rest[i] = __float_as_uint(v[i]);
#pragma unroll
  for (int k = 0; k < N; ++k) {
    i32x4 pairs;                               // the upper halves of two values each
#pragma unroll
    for (int i = 0; i < 4; ++i) pairs[i] = (int)__builtin_amdgcn_perm(rest[2 * i + 1], rest[2 * i], 0x07060302u);
    part[k] = __builtin_bit_cast(bf16x8, pairs);
    if (k + 1 < N)
#pragma unroll
      for (int i = 0; i < 8; ++i)
        rest[i] = __float_as_uint(__uint_as_float(rest[i]) - __uint_as_float(rest[i] & 0xffff0000u));
  }
}

template <class T, int QB, class Out, bool kLoose>
__global__ __launch_bounds__(64 * kSplitWaves) void k_adapter_weights(AdapterArgs p, int tiles_a, int tiles_b, int parts) {
  using E = typename T::elem;
  constexpr int kCopies = kWeightSlab / 1024;
  using Slab = std::conditional_t<kLoose, LooseAcross<E, kWeightCols, kCopies>, Copied<SlabAcross<kWeightCols, kCopies>>>;
  constexpr int NB = kWeightBlocks, XP = T::kDtype == GSQ_DT_FP16 ? 2 : 1, HP = 3;
  extern __shared__ __attribute__((aligned(16))) uint8_t smem[];
  const int tiles = (tiles_a + tiles_b) * parts;
  const int e = blockIdx.x / (unsigned)tiles, tile = blockIdx.x % (unsigned)tiles / parts, part = blockIdx.x % (unsigned)parts;
  const bool of_a = tile < tiles_a;
  const int ns = of_a ? p.I : p.O, n0 = (of_a ? tile : tile - tiles_a) * kWeightCols, j0 = part * QB * 16;
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const E* in = static_cast<const E*>(of_a ? p.x : p.dy) + n0;
  const float* hid = of_a ? p.dh : p.h;
  uint8_t* const own = smem + wave * 2 * kWeightSlab;
  f32x4 acc[QB][NB] = {};

  const auto slab_of = [&](int64_t first, int rows) {
    if constexpr (kLoose)
      return Slab(in + first * ns, ns, ns - n0, rows, 0);
    else
      return Slab(in + first * ns, (int64_t)ns * 2, ns - n0, rows, 0, lane);
  };
  struct Item {
    Slab x;
    float v[QB][8];            // hidden of rows 8 g .. and column j0 + 16 b + lane % 16
  };
  AdapterSlabs slabs(p, e, wave);
  // The next slab and its hidden are asked for, hidden first: what comes last are the copies, and only they.  Rows past
  // the last one meet zeros of x, ranks past the last one are not stored, so that others are read in their place.
  const auto ask = [&](Item& it, uint8_t* lds) {
    int64_t first;
    int rows;
    if (!slabs.next(first, rows)) return false;
    const float* from = hid + first * p.q;
#pragma unroll
    for (int b = 0; b < QB; ++b)
#pragma unroll
      for (int i = 0; i < 8; ++i)
        it.v[b][i] = from[(int64_t)min(8 * (lane >> 4) + i, rows - 1) * p.q + min(j0 + 16 * b + (lane & 15), p.q - 1)];
    __atomic_signal_fence(__ATOMIC_SEQ_CST);
    it.x = slab_of(first, rows);
    it.x.fetch(0, lds);
    return true;
  };
  // Multiplies a slab and asks for the one after the next in its place.  `other`: the next is on its way.
  const auto use = [&](Item& it, uint8_t* lds, bool other) {
    if constexpr (kLoose) {
      it.x.commit(lds);
      wait_reads();
    } else {
      __atomic_signal_fence(__ATOMIC_SEQ_CST);
      if (other)
        wait_vm<kCopies>();
      else
        wait_vm<0>();
      __atomic_signal_fence(__ATOMIC_SEQ_CST);
    }
    i32x4 f[NB];
#pragma unroll
    for (int c = 0; c < NB; ++c) f[c] = Slab::frag(lds, c * 16, 0, lane);
    bf16x8 h[QB][HP];
#pragma unroll
    for (int b = 0; b < QB; ++b) exact_parts(it.v[b], h[b]);
    wait_reads();
    const bool more = ask(it, lds);
#pragma unroll
    for (int c = 0; c < NB; ++c) {
      bf16x8 xp[XP];
      if constexpr (XP == 1) {
        xp[0] = __builtin_bit_cast(bf16x8, f[c]);
      } else {
        const f16x8 x = __builtin_bit_cast(f16x8, f[c]);
        float w[8];
#pragma unroll
        for (int i = 0; i < 8; ++i) w[i] = (float)x[i];
        exact_parts(w, xp);
      }
#pragma unroll
      for (int b = 0; b < QB; ++b)
#pragma unroll
        for (int k = HP - 1; k >= 0; --k)
#pragma unroll
          for (int y = XP - 1; y >= 0; --y)
            if (k + y < HP) acc[b][c] = Bf16::mfma(h[b][k], xp[y], acc[b][c]);
    }
    return more;
  };
  Item even{slab_of(0, 0)}, odd{slab_of(0, 0)};
  bool has_even = ask(even, own), has_odd = ask(odd, own + kWeightSlab);
  while (has_even) {
    has_even = use(even, own, has_odd);
    if (!has_odd) break;
    has_odd = use(odd, own + kWeightSlab, has_even);
  }

  // no copy is on its way any more when the sums take the slabs' place
  __atomic_signal_fence(__ATOMIC_SEQ_CST);
  wait_vm<0>();
  __atomic_signal_fence(__ATOMIC_SEQ_CST);
  // the wavefronts' sums, added in their order; a lane has rows 4 (lane / 16) + i of the rank, and of block c column
  // 16 c + lane % 16
  const float scale = of_a ? 1.f : scale_of(p, e);
  Out* out = static_cast<Out*>(of_a ? p.da : p.db) + (int64_t)e * p.q * ns;
  f32x4* const sums = reinterpret_cast<f32x4*>(smem);
#pragma unroll
  for (int b = 0; b < QB; ++b) {
    __syncthreads();
#pragma unroll
    for (int c = 0; c < NB; ++c) sums[(wave * NB + c) * 64 + lane] = acc[b][c];
    __syncthreads();
    for (int f = threadIdx.x; f < NB * 64; f += blockDim.x) {
      const int c = f / 64, l = f % 64;
      f32x4 v = {};
      for (int w = 0; w < (int)(blockDim.x >> 6); ++w) v += sums[w * NB * 64 + f];
      const int n = n0 + 16 * c + (l & 15), j = j0 + 16 * b + 4 * (l >> 4);
      if (n >= ns) continue;
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        if (j + i >= p.q) break;
        Out* to = out + (of_a ? (int64_t)(j + i) * ns + n : (int64_t)n * p.q + j + i);
        *to = (Out)(p.accumulate ? (float)*to + v[i] * scale : v[i] * scale);
      }
    }
  }
}

template <class T, int kForm, int TM, int TN, bool kLoose>
hipError_t launch_down(const AdapterArgs& p, hipStream_t s) {
  const int nk = (int)tiles_of(kForm == kForward ? p.I : p.O, kSlabRows), waves = std::min(nk, kDownWaves<TM, TN>);
  return launch_lds<k_adapter_down<T, kForm, TM, TN, kLoose>>(most_panels(p.rows, TM) * tiles_of(p.q, TN), 64 * waves,
                                                              (size_t)waves * (TM + TN) * ROW_BYTES, s, p);
}

template <class T, int kForm, bool kLoose>
hipError_t launch_rows(const AdapterArgs& p, const RowsPlan& plan, hipStream_t s) {
  hipError_t e;
  if (plan.height == 16)
    e = plan.width == 64 ? launch_down<T, kForm, 16, 64, kLoose>(p, s) : launch_down<T, kForm, 16, 16, kLoose>(p, s);
  else
    e = plan.width == 64 ? launch_down<T, kForm, 64, 64, kLoose>(p, s) : launch_down<T, kForm, 64, 16, kLoose>(p, s);
  return e;
}

constexpr int64_t kStreamBytes = (int64_t)32 << 20;   // of y, as much as the eight L2s hold

template <class T, int kForm, bool kCopied, int kBy>
hipError_t launch_up(const AdapterArgs& p, const UpPlan& plan, hipStream_t s) {
  const int ns = kForm == kForward ? p.O : p.I;
  if (!plan.steps)
    return launch_lds<k_adapter_up_few<T, kForm, kBy == kNarrow ? kNarrow : kWide>>(plan.blocks, 64 * kUpWaves, 0, s, p);
  const int chunks = (int)tiles_of(tiles_of(ns, kUpCols), plan.steps);
  if (p.q <= 32) return launch_lds<k_adapter_up<T, kForm, 1, kCopied, kBy>>(plan.blocks, 64 * kUpWaves, 0, s, p, plan.steps, chunks);
  if (p.q <= 64) return launch_lds<k_adapter_up<T, kForm, 2, kCopied, kBy>>(plan.blocks, 64 * kUpWaves, 0, s, p, plan.steps, chunks);
  return launch_lds<k_adapter_up<T, kForm, 4, kCopied, kBy>>(plan.blocks, 64 * kUpWaves, 0, s, p, plan.steps, chunks);
}

template <class T, int kForm>
hipError_t launch_both(AdapterArgs p, hipStream_t s) {
  if (p.rows.rows == 0) return hipSuccess;
  const int ks = kForm == kForward ? p.I : p.O, ns = kForm == kForward ? p.O : p.I;
  p.vector_hidden = four_at_once(p.hidden, GSQ_DT_FP32, p.q);
  const bool wide = ns % 8 == 0 && aligned16(p.out) && aligned16(p.base);
  const bool tight = kForm == kForward ? p.I % 8 == 0 && aligned16(p.x) && aligned16(p.a)
                                       : p.O % 8 == 0 && p.q % 8 == 0 && aligned16(p.dy) && aligned16(p.b);
  const bool copied = kForm == kForward ? p.q % 8 == 0 && aligned16(p.b) : p.I % 8 == 0 && aligned16(p.a);
  const RowsPlan plan = plan_adapter(p.rows.rows, p.rows.groups, p.q, (int)tiles_of(ks, kSlabRows), tight);
  const UpPlan up = plan_adapter_up(p.rows.rows, p.rows.groups, ns);
  if (!plan.height || !fits_launch(up.blocks, 64 * kUpWaves)) return hipErrorInvalidConfiguration;
  const hipError_t e = tight ? launch_rows<T, kForm, false>(p, plan, s) : launch_rows<T, kForm, true>(p, plan, s);
  if (e != hipSuccess) return e;
  if (!copied) return wide ? launch_up<T, kForm, false, kWide>(p, up, s) : launch_up<T, kForm, false, kNarrow>(p, up, s);
  if (wide && p.rows.rows * ns * 2 >= kStreamBytes) return launch_up<T, kForm, true, kStream>(p, up, s);
  return wide ? launch_up<T, kForm, true, kWide>(p, up, s) : launch_up<T, kForm, true, kNarrow>(p, up, s);
}

template <class T, class Out>
hipError_t launch_weights(const AdapterArgs& p, hipStream_t s) {
  const int64_t ta = tiles_of(p.I, kWeightCols), tb = tiles_of(p.O, kWeightCols);
  const bool tight = p.I % 8 == 0 && p.O % 8 == 0 && aligned16(p.x) && aligned16(p.dy);
  const int waves = plan_adapter_weights(p.rows.rows, p.rows.groups, p.adapters);
  const auto launch = [&](auto qb, auto loose) {
    constexpr int QB = decltype(qb)::value;
    const int64_t parts = tiles_of(p.q, 16 * QB);
    return launch_lds<k_adapter_weights<T, QB, Out, decltype(loose)::value>>(
        p.adapters * (ta + tb) * parts, 64 * waves, (size_t)waves * 2 * kWeightSlab, s, p, (int)ta, (int)tb, (int)parts);
  };
  using One = std::integral_constant<int, 1>;
  using Two = std::integral_constant<int, 2>;
  // as much of the rank together as leaves two workgroups for each of 256 CUs; slabs that pass through registers leave
  // room for one block of it
  const auto enough = [&](int qb) { return p.q > 8 * qb && p.adapters * (ta + tb) * tiles_of(p.q, 16 * qb) >= 512; };
  if (!tight) return launch(One{}, std::true_type{});
  return enough(2) ? launch(Two{}, std::false_type{}) : launch(One{}, std::false_type{});
}

}  // namespace

hipError_t launch_adapter_rows(int form, int dtype, const AdapterArgs& p, hipStream_t s) {
  const bool bf16 = dtype == GSQ_DT_BF16;
  if (form == kForward) return bf16 ? launch_both<Bf16, kForward>(p, s) : launch_both<F16, kForward>(p, s);
  return bf16 ? launch_both<Bf16, kInputGrad>(p, s) : launch_both<F16, kInputGrad>(p, s);
}

hipError_t launch_adapter_weights(int dtype, const AdapterArgs& p, hipStream_t s) {
  const bool bf16 = dtype == GSQ_DT_BF16;
  if (p.out_dtype == GSQ_DT_FP32) return bf16 ? launch_weights<Bf16, float>(p, s) : launch_weights<F16, float>(p, s);
  return bf16 ? launch_weights<Bf16, __bf16>(p, s) : launch_weights<F16, _Float16>(p, s);
}

}  // namespace gsq
