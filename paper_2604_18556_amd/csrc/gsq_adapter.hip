// Low-rank adapters of many requests: y = base + s B (A x) and its gradients, the adapter being that of the row's
// segment.
#include <hip/hip_runtime.h>

#include <algorithm>

#include "gsq_adapter.h"
#include "gsq_split.hpp"

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

// A tile of TM rows x TN of the rank, by wavefronts that share the sum.
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

template <class T, int kForm, int TM, int TN, bool kLoose>
__global__ __launch_bounds__(64 * kSplitWaves) void k_adapter_down(AdapterArgs p) {
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
// times a power of two that brings their largest value to 2^14, as its exponent would not hold both parts.
constexpr int kUpRows = 64, kUpCols = 64, kUpWaves = 4;

// Eight hidden values of a row from k on, those from q on zeros.
__device__ __forceinline__ void load_hidden(const float* row, int k, int q, float (&v)[8]) {
  if (k + 8 <= q) {
    __builtin_memcpy(v, row + k, 32);
  } else {
#pragma unroll
    for (int i = 0; i < 8; ++i) v[i] = k + i < q ? row[k + i] : 0.f;
  }
}

template <class T>
__device__ __forceinline__ void split_hidden(const float (&v)[8], float by, typename T::frag& hi, typename T::frag& lo) {
  using E = typename T::elem;
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    const float x = v[i] * by;
    const E h = (E)x;
    hi[i] = h;
    // of what is not finite there is no second part
    lo[i] = (E)(__builtin_isfinite((float)h) ? x - (float)h : 0.f);
  }
}

// 16 values of a row: as whole 16 bytes, or those that there are.
template <class E>
struct Sixteen {
  E v[16];
  __device__ __forceinline__ void load(const E* p, int n, bool whole) {
    if (whole) {
      const i32x4* q = reinterpret_cast<const i32x4*>(p);
      const i32x4 a = q[0], b = q[1];
      __builtin_memcpy(v, &a, 16);
      __builtin_memcpy(v + 8, &b, 16);
    } else {
#pragma unroll
      for (int i = 0; i < 16; ++i) v[i] = i < n ? p[i] : (E)0.f;
    }
  }
  __device__ __forceinline__ void store(E* p, int n, bool whole) const {
    if (whole) {
      i32x4 a, b;
      __builtin_memcpy(&a, v, 16);
      __builtin_memcpy(&b, v + 8, 16);
      reinterpret_cast<i32x4*>(p)[0] = a;
      reinterpret_cast<i32x4*>(p)[1] = b;
    } else {
#pragma unroll
      for (int i = 0; i < 16; ++i)
        if (i < n) p[i] = v[i];
    }
  }
};

// A wavefront's columns of the adapter's matrix, as the instructions' rows: row 4 g + c of block j is column 16 g +
// 4 j + c, so that a lane's results are 16 neighbouring columns of a row.
// B, whose rows run along the rank: straight from memory.
template <class T>
struct UpAlong {
  using E = typename T::elem;
  static constexpr size_t LDS = 0;
  const E* w;                  // the first column's row
  int cols, q;
  __device__ __forceinline__ void begin(int, uint8_t*) {}
  __device__ __forceinline__ typename T::frag frag(int k, int j) const {
    const int lane = threadIdx.x & 63, i = lane & 15, n = 16 * (i >> 2) + 4 * j + (i & 3), at = k + 8 * (lane >> 4);
    return __builtin_bit_cast(typename T::frag, load_chunk(w + (int64_t)min(n, cols - 1) * q + at, q - at));
  }
};
// A, whose rows are the rank: 64 of them and 64 columns in LDS, read by transposing reads.
template <class T, bool kLoose>
struct UpAcross {
  using E = typename T::elem;
  using Tight = SlabAcross<kUpCols, 8>;
  static constexpr size_t LDS = 64 * Tight::PITCH;
  const E* w;                  // the first column
  int64_t ld;
  int cols, q;
  uint8_t* lds = nullptr;
  __device__ __forceinline__ void begin(int k, uint8_t* own) {
    lds = own;
    if (k % kSlabRows) return;
    wait_reads();              // of the slab before
    if constexpr (kLoose) {
      LooseAcross<E, kUpCols> s(w + k * ld, ld, cols, q - k, 0);
      s.fetch(0, own);
      s.commit(own);
    } else {
      Copied<Tight> s(w + k * ld, ld * 2, cols, q - k, 0, threadIdx.x & 63);
      s.fetch(0, own);
    }
    wait_all();
  }
  __device__ __forceinline__ typename T::frag frag(int k, int j) const {
    typedef short s16x4 __attribute__((ext_vector_type(4)));
    typedef __attribute__((address_space(3))) s16x4* lds_ptr;
    const int lane = threadIdx.x & 63, r = k % kSlabRows + (lane >> 4) * 8 + ((lane & 15) >> 2);
    const uint8_t* at = lds + r * Tight::PITCH + (((lane & 3) ^ Tight::turn(r)) << 5) + j * 8;
    union { s16x4 s[2]; typename T::frag v; } u;
    u.s[0] = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_ptr)at);
    u.s[1] = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_ptr)(at + 4 * Tight::PITCH));
    return u.v;
  }
};

// SUB x 16 rows and 64 columns by one wavefront.
template <class T, int SUB, class W>
__device__ __forceinline__ void up_tile(const AdapterArgs& p, W w, float scale, int64_t first, int ms, int n0, int ns,
                                        uint8_t* own) {
  using E = typename T::elem;
  const int lane = threadIdx.x & 63, m = lane & 15, col = n0 + 16 * (lane >> 4);
  const E* base = static_cast<const E*>(p.base);
  E* out = static_cast<E*>(p.out);
  const bool whole = p.vector_out && col + 16 <= ns;
  Sixteen<E> old[SUB];
#pragma unroll
  for (int i = 0; i < SUB; ++i) {
    const int r = i * 16 + m;
    old[i].load(base + (first + r) * ns + col, base && r < ms ? ns - col : 0, whole && base && r < ms);
  }
  const float* h[SUB];
  float by[SUB];
#pragma unroll
  for (int i = 0; i < SUB; ++i) {
    h[i] = p.hidden + (first + min(i * 16 + m, ms - 1)) * p.q;
    by[i] = 1.f;
    if constexpr (T::kDtype == GSQ_DT_FP16) {
      float top = 0.f;
      for (int k = 8 * (lane >> 4); k < p.q; k += 32) {
        float v[8];
        load_hidden(h[i], k, p.q, v);
#pragma unroll
        for (int c = 0; c < 8; ++c) top = fmaxf(top, fabsf(v[c]));
      }
      top = fmaxf(top, __shfl_xor(top, 16, 64));
      top = fmaxf(top, __shfl_xor(top, 32, 64));
      // infinities (and NaN, which fmaxf leaves out) pass as they are; what is very small, as far as it goes
      if (top > 0.f && top < __builtin_huge_valf()) by[i] = exp2f((float)(13 - max((int)(__float_as_uint(top) >> 23) - 127, -100)));
    }
  }
  f32x4 acc[SUB][4] = {};
  for (int k = 0; k < p.q; k += 32) {
    w.begin(k, own);
    typename T::frag f[4];
#pragma unroll
    for (int j = 0; j < 4; ++j) f[j] = w.frag(k, j);
#pragma unroll
    for (int i = 0; i < SUB; ++i) {
      float v[8];
      load_hidden(h[i], k + 8 * (lane >> 4), p.q, v);
      typename T::frag hi, lo;
      split_hidden<T>(v, by[i], hi, lo);
#pragma unroll
      for (int j = 0; j < 4; ++j) acc[i][j] = T::mfma(f[j], hi, acc[i][j]);
#pragma unroll
      for (int j = 0; j < 4; ++j) acc[i][j] = T::mfma(f[j], lo, acc[i][j]);
    }
  }
#pragma unroll
  for (int i = 0; i < SUB; ++i) {
    const int r = i * 16 + m;
    if (r >= ms || col >= ns) continue;
    const float s = scale / by[i];           // by is a power of two
    Sixteen<E> res;
#pragma unroll
    for (int c = 0; c < 16; ++c) res.v[c] = (E)fmaf(acc[i][c / 4][c % 4], s, (float)old[i].v[c]);
    res.store(out + (first + r) * ns + col, ns - col, whole);
  }
}

// Rows without an adapter: the base, or zeros.
template <class E>
__device__ __forceinline__ void copy_base(const AdapterArgs& p, int64_t first, int ms, int n0, int ns) {
  if (p.base == p.out) return;
  const int cols = min(ns - n0, kUpCols), lane = threadIdx.x & 63;
  if (lane >= cols) return;
  for (int r = 0; r < ms; ++r) {
    const int64_t at = (first + r) * ns + n0 + lane;
    static_cast<E*>(p.out)[at] = p.base ? static_cast<const E*>(p.base)[at] : (E)0.f;
  }
}

template <class T, int kForm, bool kLoose>
__global__ __launch_bounds__(64 * kUpWaves) void k_adapter_up(AdapterArgs p) {
  using E = typename T::elem;
  using W = std::conditional_t<kForm == kForward, UpAlong<T>, UpAcross<T, kLoose>>;
  extern __shared__ __attribute__((aligned(16))) uint8_t smem[];
  const int ns = kForm == kForward ? p.O : p.I, wide = kUpCols * kUpWaves, tiles_n = (ns + wide - 1) / wide;
  PanelPlace at;
  if (!find_panel(p.rows, kUpRows, blockIdx.x / (unsigned)tiles_n, at)) return;
  int tm, tn;
  tile_at(lin_of((int)(blockIdx.x - at.before * tiles_n), at.panels * tiles_n), at.panels, tiles_n, tm, tn);
  const int64_t first = at.first + (int64_t)tm * kUpRows;
  const int ms = (int)min(at.end - first, (int64_t)kUpRows), wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int n0 = tn * wide + wave * kUpCols;
  if (n0 >= ns) return;                        // no barrier follows
  const int e = adapter_of(p, at.group);
  if (e < 0) return copy_base<E>(p, first, ms, n0, ns);
  W w;
  if constexpr (kForm == kForward) {
    w.w = static_cast<const E*>(p.b) + ((int64_t)e * p.O + n0) * p.q;
  } else {
    w.w = static_cast<const E*>(p.a) + (int64_t)e * p.q * p.I + n0;
    w.ld = p.I;
  }
  w.cols = ns - n0;
  w.q = p.q;
  const float scale = kForm == kForward ? scale_of(p, e) : 1.f;
  uint8_t* own = smem + wave * W::LDS;
  if (ms <= 16)
    up_tile<T, 1>(p, w, scale, first, ms, n0, ns, own);
  else
    up_tile<T, kUpRows / 16>(p, w, scale, first, ms, n0, ns, own);
}

// ------------------------------------------------------------------ dA, dB: sums over an adapter's rows
// fp32 matrix instructions of 16 x 16 outputs and four rows: a lane has one row of each operand, so that nothing is
// transposed, and hidden keeps its 32 bits.  A lane's 16 bytes of x (or dy) are eight columns, which go to eight
// blocks; the instructions' rows are the rank.
constexpr int kWeightWaves = 8, kWeightCols = 128;

template <class T, int QB, class Out>
__global__ __launch_bounds__(64 * kWeightWaves) void k_adapter_weights(AdapterArgs p, int tiles_a, int tiles_b, int parts) {
  using E = typename T::elem;
  __shared__ f32x4 s_sum[kWeightWaves][8][64];
  constexpr int AHEAD = 4;                     // loads of rows in flight
  const int tiles = (tiles_a + tiles_b) * parts;
  const int e = blockIdx.x / (unsigned)tiles, tile = blockIdx.x % (unsigned)tiles / parts, part = blockIdx.x % (unsigned)parts;
  const bool of_a = tile < tiles_a;
  const int ns = of_a ? p.I : p.O, n0 = (of_a ? tile : tile - tiles_a) * kWeightCols, j0 = part * QB * 16;
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const E* in = static_cast<const E*>(of_a ? p.x : p.dy);
  const float* hid = of_a ? p.dh : p.h;
  const int col = n0 + 8 * (lane & 15), left = ns - col, kk = lane >> 4;
  const int rank = j0 + (lane & 15);
  f32x4 acc[QB][8] = {};

  const auto sum_segment = [&](int segment) {
    int64_t first, end;
    group_rows(p.rows, segment, first, end);
    for (int64_t r0 = first + 4 * wave; r0 < end; r0 += 4 * kWeightWaves * AHEAD) {
      i32x4 v[AHEAD];
      float h[AHEAD][QB];
#pragma unroll
      for (int u = 0; u < AHEAD; ++u) {
        const int64_t r = r0 + u * 4 * kWeightWaves + kk;
        const bool some = r < end;
        v[u] = load_chunk(in + r * ns + col, some ? left : 0);
#pragma unroll
        for (int b = 0; b < QB; ++b) h[u][b] = some && rank + 16 * b < p.q ? hid[r * p.q + rank + 16 * b] : 0.f;
      }
#pragma unroll
      for (int u = 0; u < AHEAD; ++u) {
        E x[8];
        __builtin_memcpy(x, &v[u], 16);
#pragma unroll
        for (int c = 0; c < 8; ++c)
#pragma unroll
          for (int b = 0; b < QB; ++b)
            acc[b][c] = __builtin_amdgcn_mfma_f32_16x16x4f32(h[u][b], (float)x[c], acc[b][c], 0, 0, 0);
      }
    }
  };
  if (!p.index) {
    if (e < p.rows.groups) sum_segment(e);
  } else {
    for (int s0 = 0; s0 < p.rows.groups; s0 += 64) {
      uint64_t mine = __ballot(s0 + lane < p.rows.groups && p.index[min(s0 + lane, p.rows.groups - 1)] == e);
      while (mine) {
        sum_segment(s0 + __builtin_ctzll(mine));
        mine &= mine - 1;
      }
    }
  }

  // the wavefronts' sums, added in their order; a lane has rows 4 (lane / 16) + i of the rank, and of block c column
  // 8 (lane % 16) + c
  const float scale = of_a ? 1.f : scale_of(p, e);
  Out* out = static_cast<Out*>(of_a ? p.da : p.db) + (int64_t)e * p.q * ns;
#pragma unroll
  for (int b = 0; b < QB; ++b) {
    if (b) __syncthreads();
#pragma unroll
    for (int c = 0; c < 8; ++c) s_sum[wave][c][lane] = acc[b][c];
    __syncthreads();
    for (int f = threadIdx.x; f < 8 * 64; f += 64 * kWeightWaves) {
      const int c = f / 64, l = f % 64;
      f32x4 v = {};
#pragma unroll
      for (int w = 0; w < kWeightWaves; ++w) v += s_sum[w][c][l];
      const int n = n0 + 8 * (l & 15) + c, j = j0 + 16 * b + 4 * (l >> 4);
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
  const int nk = (int)tiles_of(kForm == kForward ? p.I : p.O, kSlabRows), waves = std::min(nk, kSplitWaves);
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

template <class T, int kForm>
hipError_t launch_both(AdapterArgs p, hipStream_t s) {
  if (p.rows.rows == 0) return hipSuccess;
  const int ks = kForm == kForward ? p.I : p.O, ns = kForm == kForward ? p.O : p.I;
  p.vector_hidden = four_at_once(p.hidden, GSQ_DT_FP32, p.q);
  p.vector_out = ns % 8 == 0 && aligned16(p.out) && aligned16(p.base);
  const bool tight = kForm == kForward ? p.I % 8 == 0 && aligned16(p.x) && aligned16(p.a)
                                       : p.O % 8 == 0 && p.q % 8 == 0 && aligned16(p.dy) && aligned16(p.b);
  const RowsPlan plan = plan_adapter(p.rows.rows, p.rows.groups, p.q, (int)tiles_of(ks, kSlabRows), tight);
  const int64_t up = most_panels(p.rows, kUpRows) * tiles_of(ns, kUpCols * kUpWaves);
  if (!plan.height || !fits_launch(up, 64 * kUpWaves)) return hipErrorInvalidConfiguration;
  const hipError_t e = tight ? launch_rows<T, kForm, false>(p, plan, s) : launch_rows<T, kForm, true>(p, plan, s);
  if (e != hipSuccess) return e;
  if constexpr (kForm == kForward)
    return launch_lds<k_adapter_up<T, kForm, false>>(up, 64 * kUpWaves, 0, s, p);
  else if (p.I % 8 == 0 && aligned16(p.a))
    return launch_lds<k_adapter_up<T, kForm, false>>(up, 64 * kUpWaves, kUpWaves * UpAcross<T, false>::LDS, s, p);
  else
    return launch_lds<k_adapter_up<T, kForm, true>>(up, 64 * kUpWaves, kUpWaves * UpAcross<T, true>::LDS, s, p);
}

template <class T, class Out>
hipError_t launch_weights(const AdapterArgs& p, hipStream_t s) {
  const int64_t ta = tiles_of(p.I, kWeightCols), tb = tiles_of(p.O, kWeightCols);
  const auto launch = [&](auto qb) {
    constexpr int QB = decltype(qb)::value;
    const int64_t parts = tiles_of(p.q, 16 * QB);
    return launch_lds<k_adapter_weights<T, QB, Out>>(p.adapters * (ta + tb) * parts, 64 * kWeightWaves, 0, s, p, (int)ta,
                                                     (int)tb, (int)parts);
  };
  if (p.q <= 16) return launch(std::integral_constant<int, 1>{});
  if (p.q <= 32) return launch(std::integral_constant<int, 2>{});
  return launch(std::integral_constant<int, 4>{});
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
