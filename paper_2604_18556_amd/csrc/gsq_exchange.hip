// Rows to the experts and back: tokens copied into the experts' order, the experts' rows summed with weights, and the
// gradients of the sum.  All three are bound by memory: a thread has 16 bytes of a row, or several 16 bytes that lie
// the threads of a row apart.
#include <hip/hip_runtime.h>

#include <algorithm>

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
  int32_t K, C, shift;         // 2^shift threads have a token
};

// 16 bytes of a row from any address, as far as there are that many.
template <class E>
struct Piece {
  static constexpr int PER = 16 / (int)sizeof(E);
  E v[PER];
  __device__ __forceinline__ void load(const E* row, int c, int cols) {
    if (c + PER <= cols) {
      __builtin_memcpy(v, row + c, 16);
    } else {
#pragma unroll
      for (int i = 0; i < PER; ++i) v[i] = c + i < cols ? row[c + i] : (E)0.f;
    }
  }
  __device__ __forceinline__ void store(E* row, int c, int cols) const {
    if (c + PER <= cols) {
      __builtin_memcpy(row + c, v, 16);
    } else {
#pragma unroll
      for (int i = 0; i < PER; ++i)
        if (c + i < cols) row[c + i] = v[i];
    }
  }
};

// The token of this thread in round `n` of the grid, and its place among the token's threads.
struct Place {
  int64_t token, step;
  int lane, lanes;
  __device__ __forceinline__ explicit Place(const ExchangeArgs& p)
      : token(((int64_t)blockIdx.x * blockDim.x + threadIdx.x) >> p.shift),
        step((int64_t)gridDim.x * blockDim.x >> p.shift), lane(threadIdx.x & ((1 << p.shift) - 1)), lanes(1 << p.shift) {}
};

template <class E>
__global__ __launch_bounds__(256) void k_dispatch(ExchangeArgs p) {
  constexpr int PER = Piece<E>::PER, HELD = 4;
  const Place at(p);
  for (int64_t t = at.token; t < p.tokens; t += at.step) {
    const E* x = static_cast<const E*>(p.in) + t * p.C;
    const int32_t* slots = p.slots + t * p.K;
    for (int c0 = at.lane * PER; c0 < p.C; c0 += at.lanes * PER * HELD) {
      Piece<E> v[HELD];
#pragma unroll
      for (int h = 0; h < HELD; ++h) v[h].load(x, min(c0 + h * at.lanes * PER, p.C), p.C);
      for (int k = 0; k < p.K; ++k) {
        const int64_t slot = slots[k];
        if (slot < 0 || slot >= p.n_rows) continue;
        E* out = static_cast<E*>(p.out) + slot * p.C;
#pragma unroll
        for (int h = 0; h < HELD; ++h) v[h].store(out, min(c0 + h * at.lanes * PER, p.C), p.C);
      }
    }
  }
}

constexpr int kAtOnce = 8;     // rows of a token that are asked for together

template <class E, bool kWeighted>
__global__ __launch_bounds__(256) void k_combine(ExchangeArgs p) {
  constexpr int PER = Piece<E>::PER;
  const Place at(p);
  for (int64_t t = at.token; t < p.tokens; t += at.step) {
    const int32_t* slots = p.slots + t * p.K;
    const float* weights = p.weights + t * p.K;
    for (int c = at.lane * PER; c < p.C; c += at.lanes * PER) {
      float sum[PER] = {};
      for (int k0 = 0; k0 < p.K; k0 += kAtOnce) {
        Piece<E> v[kAtOnce];
        float w[kAtOnce];
#pragma unroll
        for (int u = 0; u < kAtOnce; ++u) {
          const int64_t slot = k0 + u < p.K ? slots[k0 + u] : -1;
          w[u] = kWeighted && k0 + u < p.K ? weights[k0 + u] : k0 + u < p.K ? 1.f : 0.f;
#pragma unroll
          for (int i = 0; i < PER; ++i) v[u].v[i] = (E)0.f;
          if (slot >= 0 && slot < p.n_rows) v[u].load(static_cast<const E*>(p.in) + slot * p.C, c, p.C);
        }
#pragma unroll
        for (int u = 0; u < kAtOnce; ++u)
#pragma unroll
          for (int i = 0; i < PER; ++i) sum[i] = fmaf(w[u], (float)v[u].v[i], sum[i]);
      }
      Piece<E> r;
#pragma unroll
      for (int i = 0; i < PER; ++i) r.v[i] = (E)sum[i];
      r.store(static_cast<E*>(p.out) + t * p.C, c, p.C);
    }
  }
}

// The sum over a token's threads, in a fixed order; every thread of the workgroup calls it.
__device__ __forceinline__ float token_sum(float v, int lanes, float* part) {
  for (int d = 1; d < min(lanes, 64); d <<= 1) v += __shfl_xor(v, d, 64);
  if (lanes <= 64) return v;
  __syncthreads();
  if ((threadIdx.x & 63) == 0) part[threadIdx.x >> 6] = v;
  __syncthreads();
  const int waves = lanes >> 6, first = (threadIdx.x >> 6) / waves * waves;
  float all = 0.f;
  for (int w = 0; w < waves; ++w) all += part[first + w];
  return all;
}

template <class E>
__global__ __launch_bounds__(256) void k_combine_grad(ExchangeArgs p) {
  constexpr int PER = Piece<E>::PER;
  __shared__ float part[4];
  const Place at(p);
  // every thread of a workgroup makes as many rounds as its first
  for (int64_t t0 = ((int64_t)blockIdx.x * blockDim.x) >> p.shift; t0 < p.tokens; t0 += at.step) {
    const int64_t t = t0 + (threadIdx.x >> p.shift);
    const bool live = t < p.tokens;
    const int64_t tt = live ? t : p.tokens - 1;
    const int32_t* slots = p.slots + tt * p.K;
    const float* weights = p.weights + tt * p.K;
    for (int k0 = 0; k0 < p.K; k0 += kAtOnce) {
      int64_t slot[kAtOnce];
      float w[kAtOnce], dot[kAtOnce];
#pragma unroll
      for (int u = 0; u < kAtOnce; ++u) {
        slot[u] = k0 + u < p.K && live ? slots[k0 + u] : -1;
        if (slot[u] >= p.n_rows) slot[u] = -1;
        w[u] = k0 + u < p.K ? weights[k0 + u] : 0.f;
        dot[u] = 0.f;
      }
      for (int c = at.lane * PER; c < p.C; c += at.lanes * PER) {
        Piece<E> d, v[kAtOnce];
        d.load(static_cast<const E*>(p.in) + tt * p.C, c, p.C);
#pragma unroll
        for (int u = 0; u < kAtOnce; ++u)
          if (slot[u] >= 0) v[u].load(static_cast<const E*>(p.rows) + slot[u] * p.C, c, p.C);
#pragma unroll
        for (int u = 0; u < kAtOnce; ++u) {
          if (slot[u] < 0) continue;
          Piece<E> r;
#pragma unroll
          for (int i = 0; i < PER; ++i) {
            dot[u] = fmaf((float)d.v[i], (float)v[u].v[i], dot[u]);
            r.v[i] = (E)(w[u] * (float)d.v[i]);
          }
          r.store(static_cast<E*>(p.out) + slot[u] * p.C, c, p.C);
        }
      }
#pragma unroll
      for (int u = 0; u < kAtOnce; ++u) {
        if (k0 + u >= p.K) break;
        const float all = token_sum(dot[u], at.lanes, part);
        if (live && at.lane == 0) p.dweights[t * p.K + k0 + u] = all;
      }
    }
  }
}

template <class F>
hipError_t with_type(int dtype, F f) {
  if (dtype == GSQ_DT_BF16) return f(__bf16{});
  if (dtype == GSQ_DT_FP16) return f(_Float16{});
  return f(float{});
}

// Threads of a token: as many as its row has pieces of 16 bytes, up to a workgroup.
ExchangeArgs exchange_args(const gsq_exchange& g, const void* in, const int32_t* slots, void* out) {
  ExchangeArgs p{};
  p.in = in;
  p.slots = slots;
  p.out = out;
  p.tokens = g.tokens;
  p.n_rows = g.rows;
  p.K = g.copies;
  p.C = g.cols;
  const int64_t pieces = tiles_of(g.cols, g.dtype == GSQ_DT_FP32 ? 4 : 8);
  while (p.shift < 8 && ((int64_t)1 << p.shift) < pieces) ++p.shift;
  return p;
}
unsigned exchange_blocks(const ExchangeArgs& p) {
  return (unsigned)std::min<int64_t>(tiles_of(p.tokens, 256 >> p.shift), 1 << 20);
}

}  // namespace

hipError_t launch_dispatch(const gsq_exchange& g, const void* x, const int32_t* slots, void* out, hipStream_t s) {
  if (g.tokens == 0) return hipSuccess;
  const ExchangeArgs p = exchange_args(g, x, slots, out);
  return with_type(g.dtype, [&](auto type) {
    k_dispatch<decltype(type)><<<exchange_blocks(p), 256, 0, s>>>(p);
    return hipGetLastError();
  });
}

hipError_t launch_combine(const gsq_exchange& g, const void* rows, const int32_t* slots, const float* weights, void* out,
                          hipStream_t s) {
  if (g.tokens == 0) return hipSuccess;
  ExchangeArgs p = exchange_args(g, rows, slots, out);
  p.weights = weights;
  return with_type(g.dtype, [&](auto type) {
    if (weights)
      k_combine<decltype(type), true><<<exchange_blocks(p), 256, 0, s>>>(p);
    else
      k_combine<decltype(type), false><<<exchange_blocks(p), 256, 0, s>>>(p);
    return hipGetLastError();
  });
}

hipError_t launch_combine_grad(const gsq_exchange& g, const void* dout, const void* rows, const int32_t* slots,
                               const float* weights, void* drows, float* dweights, hipStream_t s) {
  if (g.tokens == 0) return hipSuccess;
  ExchangeArgs p = exchange_args(g, dout, slots, drows);
  p.rows = rows;
  p.weights = weights;
  p.dweights = dweights;
  return with_type(g.dtype, [&](auto type) {
    k_combine_grad<decltype(type)><<<exchange_blocks(p), 256, 0, s>>>(p);
    return hipGetLastError();
  });
}

}  // namespace gsq
