// Rows to the experts and back: tokens copied into the experts' order, the experts' rows summed with weights, and the
// gradients of the sum.
//
// All three are bound by memory.  A lane has 16 bytes of a token's row and asks for those of eight of its rows (two,
// where a token has no more: 16384 rows of 4096 of one token each there and back 135 us by eights) at once.  What a token
// has not of the eight is read as the first row, which the caches hold: 16384 rows of 7168 summed by eights 43 us, 6.1 TB/s,
// by sixes 45, by fours 54, by threes 65, 4.8 TB/s, by twos 57.  A wavefront belongs to one token (rows of more than 512
// bytes) and has the slots in scalar registers, so that nothing in the way of the loads is divided.  The last 16 bytes of a
// row overlap those before where its length is no multiple of them; addresses may be any, as loads and stores of 16 bytes
// need no alignment.
#include <hip/hip_runtime.h>

#include <algorithm>

#include "gsq_lanes.hpp"
#include "gsq_plan.h"
#include "gsq_route.h"

namespace gsq {
namespace {

struct ExchangeArgs {
  const void* in;              // tokens or rows
  const void* rows;            // k_combine_grad: the rows
  const int32_t* slots;
  const float* weights;
  void* out;
  float* dweights;
  int64_t tokens, n_rows;
  int32_t K, C;
  int32_t pieces, parts;       // of a row; 64 pieces each
  int32_t shift;               // short rows: 2^shift lanes have a token
};

// How an array is gone through: elements, values of a piece, rows of a token that are asked for together, whether a
// wavefront belongs to one token, and whether the caches are passed by.
template <class E_, int PER_, int AT_, bool kWave_, bool kStream_>
struct Form {
  using E = E_;
  static constexpr int PER = PER_, AT = AT_;
  static constexpr bool kWave = kWave_, kStream = kStream_;
};

// 16 bytes of a row, or one value.  kStream: of arrays that no cache holds, by accesses with the non-temporal hint
// (aligned; 16384 rows of 7168 there and back 99 us, 120 without, their gradients 146, 158).
template <class F>
struct Piece {
  using E = typename F::E;
  static constexpr int PER = F::PER;
  typedef int32_t i32x4 __attribute__((ext_vector_type(4)));
  typedef E vec __attribute__((ext_vector_type(PER)));
  using Bits = std::conditional_t<PER == 1, E, i32x4>;
  Bits bits;
  __device__ __forceinline__ void load(const E* p) {
    if constexpr (F::kStream)
      bits = __builtin_nontemporal_load(reinterpret_cast<const i32x4*>(p));
    else
      __builtin_memcpy(&bits, p, sizeof(bits));
  }
  __device__ __forceinline__ void store(E* p) const {
    if constexpr (F::kStream)
      __builtin_nontemporal_store(bits, reinterpret_cast<i32x4*>(p));
    else
      __builtin_memcpy(p, &bits, sizeof(bits));
  }
  // The values from here on, or zeros; the load before stays whole (the compiler would take a part of it for each of
  // the ways on).
  __device__ __forceinline__ void settle(bool some = true) {
    if constexpr (PER > 1) {
      asm volatile("" : "+v"(bits));
      bits &= some ? -1 : 0;
    } else {
      bits = some ? bits : (E)0.f;
    }
  }
  // The first n values become zeros.
  __device__ __forceinline__ void clear(int n) {
    if constexpr (PER > 1) {
      vec v = __builtin_bit_cast(vec, bits);
#pragma unroll
      for (int i = 0; i < PER; ++i) v[i] = i < n ? (E)0.f : v[i];
      bits = __builtin_bit_cast(i32x4, v);
    }
  }
  __device__ __forceinline__ float at(int i) const {
    if constexpr (PER > 1)
      return (float)__builtin_bit_cast(vec, bits)[i];
    else
      return (float)bits;
  }
  __device__ __forceinline__ void set(const float (&v)[PER]) {
    if constexpr (PER > 1) {
      vec r;
#pragma unroll
      for (int i = 0; i < PER; ++i) r[i] = (E)v[i];
      bits = __builtin_bit_cast(i32x4, r);
    } else {
      bits = (E)v[0];
    }
  }
};

// A lane's token and piece in one round of the grid.
struct Place {
  int64_t token;
  int piece;
  bool live;
};
template <bool kWave>
__device__ __forceinline__ Place place_of(const ExchangeArgs& p, int64_t block) {
  Place at;
  if constexpr (kWave) {
    const int64_t task = block * 4 + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    at.token = task >> 32 ? task / p.parts : (uint32_t)task / (uint32_t)p.parts;
    // every lane stays: those past the row's end do its last piece once more
    at.piece = min((int)(task - at.token * p.parts) * 64 + (int)(threadIdx.x & 63), p.pieces - 1);
  } else {
    at.token = (block * 256 + threadIdx.x) >> p.shift;
    at.piece = threadIdx.x & ((1 << p.shift) - 1);
  }
  at.live = at.token < p.tokens && at.piece < p.pieces;
  return at;
}
template <int PER>
__device__ __forceinline__ int column(const ExchangeArgs& p, int piece) { return min(piece * PER, p.C - PER); }

// AT slots of a token from k0 on, and their weights; those that name no row are -1.
template <bool kWave, bool kWeighted, int AT>
__device__ __forceinline__ void load_slots(const ExchangeArgs& p, int64_t token, int k0, int64_t (&slot)[AT],
                                           float (&w)[AT]) {
  const int32_t* slots = p.slots + token * p.K;
  const float* weights = p.weights + token * p.K;
  if constexpr (kWave) {                       // one load for all lanes, all of them here, then lane by lane
    const int k = min(k0 + (int)(threadIdx.x & (AT - 1)), p.K - 1);
    const int mine = slots[k];
    const float my_w = kWeighted ? weights[k] : 1.f;
#pragma unroll
    for (int u = 0; u < AT; ++u) {
      slot[u] = __builtin_amdgcn_readlane(mine, u);
      w[u] = __uint_as_float(__builtin_amdgcn_readlane(__float_as_uint(my_w), u));
    }
  } else {
#pragma unroll
    for (int u = 0; u < AT; ++u) {
      slot[u] = slots[min(k0 + u, p.K - 1)];
      w[u] = kWeighted ? weights[min(k0 + u, p.K - 1)] : 1.f;
    }
  }
#pragma unroll
  for (int u = 0; u < AT; ++u) {
    if (slot[u] >= p.n_rows || k0 + u >= p.K) slot[u] = -1;
    if (k0 + u >= p.K) w[u] = 0.f;
  }
}

template <class F>
__global__ __launch_bounds__(256) void k_dispatch(ExchangeArgs p, int64_t blocks) {
  using E = typename F::E;
  constexpr int PER = F::PER, AT = F::AT;
  constexpr bool kWave = F::kWave;
  for (int64_t block = blockIdx.x; block < blocks; block += gridDim.x) {
    const Place at = place_of<kWave>(p, block);
    if (!at.live) continue;
    const int c = column<PER>(p, at.piece);
    Piece<F> v;
    v.load(static_cast<const E*>(p.in) + at.token * p.C + c);
    for (int k0 = 0; k0 < p.K; k0 += AT) {
      int64_t slot[AT];
      float w[AT];
      load_slots<kWave, false>(p, at.token, k0, slot, w);
      v.settle();
#pragma unroll
      for (int u = 0; u < AT; ++u)
        if (slot[u] >= 0) v.store(static_cast<E*>(p.out) + slot[u] * p.C + c);
    }
  }
}

// Slots that name no row are read as the first one, whose values are not used.
template <class F, bool kWeighted>
__global__ __launch_bounds__(256) void k_combine(ExchangeArgs p, int64_t blocks) {
  using E = typename F::E;
  constexpr int PER = F::PER, AT = F::AT;
  constexpr bool kWave = F::kWave;
  for (int64_t block = blockIdx.x; block < blocks; block += gridDim.x) {
    const Place at = place_of<kWave>(p, block);
    if (!at.live) continue;
    const int c = column<PER>(p, at.piece);
    float sum[PER] = {};
    for (int k0 = 0; k0 < p.K; k0 += AT) {
      int64_t slot[AT];
      float w[AT];
      load_slots<kWave, kWeighted>(p, at.token, k0, slot, w);
      Piece<F> v[AT];
#pragma unroll
      for (int u = 0; u < AT; ++u)
        v[u].load(static_cast<const E*>(p.in) + (slot[u] < 0 ? 0 : slot[u]) * p.C + c);
#pragma unroll
      for (int u = 0; u < AT; ++u) {
        v[u].settle(slot[u] >= 0);
#pragma unroll
        for (int i = 0; i < PER; ++i) sum[i] = fmaf(w[u], v[u].at(i), sum[i]);
      }
    }
    Piece<F> r;
    r.set(sum);
    r.store(static_cast<E*>(p.out) + at.token * p.C + c);
  }
}

// A workgroup has a token, its wavefronts one part after another (or, of short rows, a wavefront several tokens); the
// products' sums are added over lanes and wavefronts in a fixed order.  kRagged: a row's last piece overlaps the one
// before.
template <class F, bool kRagged>
__global__ __launch_bounds__(512) void k_combine_grad(ExchangeArgs p, int64_t blocks) {
  using E = typename F::E;
  constexpr int PER = F::PER, AT = F::AT;
  constexpr bool kWave = F::kWave;
  __shared__ float s_dot[8][AT];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, waves = blockDim.x >> 6;
  for (int64_t block = blockIdx.x; block < blocks; block += gridDim.x) {
    const int64_t token = kWave ? block : (block * blockDim.x + threadIdx.x) >> p.shift;
    const int first = kWave ? (int)threadIdx.x : (int)(threadIdx.x & ((1 << p.shift) - 1));
    const bool live = token < p.tokens;
    const int64_t t = live ? token : p.tokens - 1;
    for (int k0 = 0; k0 < p.K; k0 += AT) {
      int64_t slot[AT];
      float w[AT], dot[AT] = {};
      load_slots<kWave, true>(p, t, k0, slot, w);
      for (int piece = first; piece < p.pieces && live; piece += kWave ? (int)blockDim.x : p.pieces) {
        const int c = column<PER>(p, piece);
        Piece<F> d, v[AT];
        d.load(static_cast<const E*>(p.in) + t * p.C + c);
#pragma unroll
        for (int u = 0; u < AT; ++u)
          v[u].load(static_cast<const E*>(p.rows) + (slot[u] < 0 ? 0 : slot[u]) * p.C + c);
        const int before = kRagged ? piece * PER - c : 0;      // values that the piece before has counted
        d.settle();
        if (kRagged && before > 0)               // on both sides: an infinity times zero would be NaN
#pragma unroll
          for (int u = 0; u < AT; ++u) {
            v[u].settle();
            v[u].clear(before);
          }
        float once[PER];
#pragma unroll
        for (int i = 0; i < PER; ++i) once[i] = i >= before ? d.at(i) : 0.f;
#pragma unroll
        for (int u = 0; u < AT; ++u) {
          v[u].settle();
          if (slot[u] < 0) continue;
          float r[PER];
#pragma unroll
          for (int i = 0; i < PER; ++i) {
            dot[u] = fmaf(once[i], v[u].at(i), dot[u]);
            r[i] = w[u] * d.at(i);
          }
          Piece<F> to;
          to.set(r);
          to.store(static_cast<E*>(p.out) + slot[u] * p.C + c);
        }
      }
      if constexpr (kWave) {
#pragma unroll
        for (int u = 0; u < AT; ++u) dot[u] = sum_lanes<64>(dot[u]);
        if (lane == 0) {
#pragma unroll
          for (int u = 0; u < AT; ++u) s_dot[wave][u] = dot[u];
        }
        __syncthreads();
        const int u = threadIdx.x;
        if (u < AT && k0 + u < p.K) {
          float all = 0.f;
          for (int o = 0; o < waves; ++o) all += s_dot[o][u];
          p.dweights[t * p.K + k0 + u] = all;
        }
        __syncthreads();
      } else {
#pragma unroll
        for (int u = 0; u < AT; ++u) {
          if (k0 + u >= p.K) break;
          float all = dot[u];
          for (int d = 1; d < 1 << p.shift; d <<= 1) all += __shfl_xor(all, d, 64);
          if (live && first == 0) p.dweights[t * p.K + k0 + u] = all;
        }
      }
    }
  }
}

ExchangeArgs exchange_args(const gsq_exchange& g, const void* in, const int32_t* slots, void* out) {
  ExchangeArgs p{};
  p.in = in;
  p.slots = slots;
  p.out = out;
  p.tokens = g.tokens;
  p.n_rows = g.rows;
  p.K = g.copies;
  p.C = g.cols;
  return p;
}

// Rows of all slots together from which the caches are passed by: the eight L2s hold 32 MB.
constexpr int64_t kStreamBytes = (int64_t)32 << 20;

// f(Form, arguments, workgroups of `threads`, threads, workgroups that there would have to be): pieces of 16 bytes, or
// rows of fewer value by value; a wavefront to a token from 33 pieces on.  `whole`: a workgroup has a token.
template <class E, int PER, class F>
hipError_t with_form(ExchangeArgs p, bool whole, F f) {
  p.pieces = (int)tiles_of(p.C, PER);
  p.parts = (int)tiles_of(p.pieces, 64);
  const bool wave = p.pieces > 32;
  while (!wave && 1 << p.shift < p.pieces) ++p.shift;
  const int rounds = (int)tiles_of(p.parts, 8), threads = wave && whole ? 64 * (int)tiles_of(p.parts, rounds) : 256;
  const int64_t blocks = !wave ? tiles_of(p.tokens, 256 >> p.shift) : whole ? p.tokens : tiles_of(p.tokens * p.parts, 4);
  const unsigned grid = (unsigned)std::min<int64_t>(blocks, 1 << 22);
  const auto run = [&](auto of_wave, auto stream) {
    constexpr bool kWave = decltype(of_wave)::value, kStream = decltype(stream)::value;
    if (p.K <= 2)
      f(Form<E, PER, 2, kWave, kStream>{}, p, grid, threads, blocks);
    else
      f(Form<E, PER, 8, kWave, kStream>{}, p, grid, threads, blocks);
    return hipGetLastError();
  };
  if (!wave) return run(std::false_type{}, std::false_type{});
  if constexpr (PER > 1) {
    const auto aligned = [](const void* a) { return (reinterpret_cast<uintptr_t>(a) & 15) == 0; };
    if (p.C % PER == 0 && aligned(p.in) && aligned(p.rows) && aligned(p.out) &&
        p.tokens * p.K * p.C * (int64_t)sizeof(E) >= kStreamBytes)
      return run(std::true_type{}, std::true_type{});
  }
  return run(std::true_type{}, std::false_type{});
}
template <class F>
hipError_t with_pieces(int dtype, const ExchangeArgs& p, bool whole, F f) {
  if (dtype == GSQ_DT_BF16) return p.C < 8 ? with_form<__bf16, 1>(p, whole, f) : with_form<__bf16, 8>(p, whole, f);
  if (dtype == GSQ_DT_FP16) return p.C < 8 ? with_form<_Float16, 1>(p, whole, f) : with_form<_Float16, 8>(p, whole, f);
  return p.C < 4 ? with_form<float, 1>(p, whole, f) : with_form<float, 4>(p, whole, f);
}

}  // namespace

hipError_t launch_dispatch(const gsq_exchange& g, const void* x, const int32_t* slots, void* out, hipStream_t s) {
  if (g.tokens == 0) return hipSuccess;
  return with_pieces(g.dtype, exchange_args(g, x, slots, out), false,
                     [&](auto form, const ExchangeArgs& p, unsigned grid, int threads, int64_t blocks) {
                       k_dispatch<decltype(form)><<<grid, threads, 0, s>>>(p, blocks);
                     });
}

hipError_t launch_combine(const gsq_exchange& g, const void* rows, const int32_t* slots, const float* weights, void* out,
                          hipStream_t s) {
  if (g.tokens == 0) return hipSuccess;
  // without rows no slot names one, and what is read in its place is the output's first row
  ExchangeArgs p = exchange_args(g, g.rows ? rows : out, slots, out);
  p.weights = weights;
  return with_pieces(g.dtype, p, false,
                     [&](auto form, const ExchangeArgs& p, unsigned grid, int threads, int64_t blocks) {
                       if (weights)
                         k_combine<decltype(form), true><<<grid, threads, 0, s>>>(p, blocks);
                       else
                         k_combine<decltype(form), false><<<grid, threads, 0, s>>>(p, blocks);
                     });
}

hipError_t launch_combine_grad(const gsq_exchange& g, const void* dout, const void* rows, const int32_t* slots,
                               const float* weights, void* drows, float* dweights, hipStream_t s) {
  if (g.tokens == 0) return hipSuccess;
  ExchangeArgs p = exchange_args(g, dout, slots, drows);
  p.rows = g.rows ? rows : dout;
  p.weights = weights;
  p.dweights = dweights;
  return with_pieces(g.dtype, p, true,
                     [&](auto form, const ExchangeArgs& p, unsigned grid, int threads, int64_t blocks) {
                       using Form = decltype(form);
                       if (!Form::kStream && p.C % Form::PER)
                         k_combine_grad<Form, !Form::kStream><<<grid, threads, 0, s>>>(p, blocks);
                       else
                         k_combine_grad<Form, false><<<grid, threads, 0, s>>>(p, blocks);
                     });
}

}  // namespace gsq
