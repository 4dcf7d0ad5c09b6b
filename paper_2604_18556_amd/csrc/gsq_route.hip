// Experts of tokens: their choice and weights from the logits, the logits' gradient, and the order that brings each
// expert's rows together.
//
// A token's logits stay in the registers of the lanes that share it.  What bounds these kernels is latency: 16384 tokens
// of 64 experts are 2 MB, and take 6.6 us to choose (vector units busy 0.24) and 12 us in three launches to order; 64
// tokens of 256 grouped experts take 6.8 and 3.9 us.
#include <hip/hip_runtime.h>

#include <algorithm>
#include <type_traits>

#include "gsq_lanes.hpp"
#include "gsq_plan.h"
#include "gsq_route.h"

namespace gsq {
namespace {

constexpr float kLowest = -__builtin_huge_valf();

struct RouteArgs {
  const void* logits;
  const float* bias;
  int32_t* experts;            // k_route_grad reads them
  float* weights;
  const float* dweights;
  void* dlogits;
  int64_t tokens;
  int32_t E, K, groups, top_groups;
  uint32_t group_size, group_inv;   // expert e is in group (e group_inv) >> 20
  int32_t sigmoid, top2, renormalise;
  float scale;
  int32_t dtype;               // of the logits
  int32_t group_share;         // 2^group_share lanes look at a group
};

// A lane's PER neighbouring logits of a token, as fp32; those past the last one are -infinity.
template <class E, int PER>
__device__ __forceinline__ void load_logits_of(const E* row, int E_, int e0, float (&l)[PER]) {
  E v[PER];
  if (e0 + PER <= E_) {
    __builtin_memcpy(v, row + e0, sizeof(v));
#pragma unroll
    for (int j = 0; j < PER; ++j) l[j] = (float)v[j];
  } else {
#pragma unroll
    for (int j = 0; j < PER; ++j) l[j] = e0 + j < E_ ? (float)row[e0 + j] : kLowest;
  }
}
template <int PER>
__device__ __forceinline__ void load_logits(const RouteArgs& p, int64_t token, int e0, float (&l)[PER]) {
  if (p.dtype == GSQ_DT_BF16)
    load_logits_of(static_cast<const __bf16*>(p.logits) + token * p.E, p.E, e0, l);
  else if (p.dtype == GSQ_DT_FP16)
    load_logits_of(static_cast<const _Float16*>(p.logits) + token * p.E, p.E, e0, l);
  else
    load_logits_of(static_cast<const float*>(p.logits) + token * p.E, p.E, e0, l);
}
template <class E, int PER>
__device__ __forceinline__ void store_gradient_as(E* row, int E_, int e0, const float (&d)[PER]) {
  E v[PER];
#pragma unroll
  for (int j = 0; j < PER; ++j) v[j] = (E)d[j];
  if (e0 + PER <= E_) {
    __builtin_memcpy(row + e0, v, sizeof(v));
  } else {
#pragma unroll
    for (int j = 0; j < PER; ++j)
      if (e0 + j < E_) row[e0 + j] = v[j];
  }
}

// LANES lanes have a token, PER neighbouring experts each.  Keys are compared in 64 bits where a bias is added (two
// experts' sums may differ in what 32 bits lose), and as the logits themselves where it is not.
template <class Key, int LANES, int PER>
__global__ __launch_bounds__(64) void k_route(RouteArgs p) {
  constexpr int TOKENS = 64 / LANES, MOST = LANES * PER;
  constexpr bool kBias = std::is_same<Key, double>::value;
  constexpr int PITCH = MOST + MOST / 16;   // so that groups of 16, 32 .. experts begin on different banks
  __shared__ float s_logit[TOKENS][MOST];
  __shared__ int s_chosen[TOKENS][GSQ_MAX_TOP_K];
  __shared__ double s_group[TOKENS][GSQ_MAX_EXPERT_GROUPS];
  __shared__ uint8_t s_kept[TOKENS][GSQ_MAX_EXPERT_GROUPS];
  extern __shared__ double s_value[];       // with groups: TOKENS x PITCH
  const int tid = threadIdx.x, lane = tid % LANES, sub = tid / LANES, e0 = lane * PER;
  const int64_t token = (int64_t)blockIdx.x * TOKENS + sub;
  const bool live = token < p.tokens;

  float l[PER];
  load_logits<PER>(p, live ? token : p.tokens - 1, e0, l);
  float top = kLowest, wrong = 0.f;
#pragma unroll
  for (int j = 0; j < PER; ++j) {
    s_logit[sub][e0 + j] = l[j];
    if (l[j] != l[j] || (!p.sigmoid && l[j] == -kLowest)) wrong = 1.f;
    top = fmaxf(top, l[j]);
  }
  top = max_lanes<LANES>(top);
  wrong = max_lanes<LANES>(wrong);
  if (top == kLowest) top = 0.f;            // no expert: every exponential is zero

  // the scores: softmax's sum in 32 bits serves the weights, keys and groups take 64
  double total = 1.0;
  double score[PER];
  const bool scored = kBias || p.groups > 1;
  if (scored) {
    double sum = 0.0;
#pragma unroll
    for (int j = 0; j < PER; ++j) {
      score[j] = p.sigmoid ? 1.0 / (1.0 + exp(-(double)l[j])) : exp((double)l[j] - (double)top);
      sum += score[j];
    }
    if (!p.sigmoid) {
      total = sum_lanes<LANES>(sum);
      const double inv = total > 0.0 ? 1.0 / total : 0.0;
#pragma unroll
      for (int j = 0; j < PER; ++j) score[j] *= inv;
    }
  } else if (!p.sigmoid && !p.renormalise) {
    float sum = 0.f;
#pragma unroll
    for (int j = 0; j < PER; ++j) sum += expf(l[j] - top);
    total = sum_lanes<LANES>(sum);
  }

  Key key[PER];
#pragma unroll
  for (int j = 0; j < PER; ++j) {
    if constexpr (kBias) {
      score[j] += e0 + j < p.E ? (double)p.bias[e0 + j] : 0.0;
      key[j] = l[j] > kLowest && score[j] == score[j] ? score[j] : (double)kLowest;
    } else {
      key[j] = l[j] == l[j] ? l[j] : kLowest;
    }
  }

  if (p.groups > 1) {
    double* value = s_value + sub * PITCH;
#pragma unroll
    for (int j = 0; j < PER; ++j)
      value[(e0 + j) + (e0 + j) / 16] = l[j] > kLowest && score[j] == score[j] ? score[j] : (double)kLowest;
    __syncthreads();
    // 2^share lanes to a group, or groups one after another
    const int share = p.group_share, mates = 1 << share;
    for (int g = lane >> share; g < p.groups; g += LANES >> share) {
      double best = kLowest, second = kLowest;
      for (int e = lane & (mates - 1); e < (int)p.group_size; e += mates) {
        const int i = g * p.group_size + e;
        const double v = value[i + i / 16];
        second = max_of(second, v > best ? best : v);
        best = max_of(best, v);
      }
      for (int d = 1; d < mates; d <<= 1) {
        const double b = __shfl_xor(best, d, 64), s = __shfl_xor(second, d, 64);
        second = max_of(max_of(second, s), b > best ? best : b);
        best = max_of(best, b);
      }
      if ((lane & (mates - 1)) == 0) s_group[sub][g] = p.top2 && second > (double)kLowest ? best + second : best;
    }
    __syncthreads();
    for (int g = lane; g < p.groups; g += LANES) {
      const double mine = s_group[sub][g];
      int before = 0;
#pragma unroll 4
      for (int h = 0; h < p.groups; ++h) {
        const double other = s_group[sub][h];
        before += other > mine || (other == mine && h < g);
      }
      s_kept[sub][g] = before < p.top_groups;
    }
    __syncthreads();
#pragma unroll
    for (int j = 0; j < PER; ++j)
      if (e0 + j < p.E && !s_kept[sub][(e0 + j) * p.group_inv >> 20]) key[j] = kLowest;
  }

  // the best of those left, K times; lanes and their experts are in order, so that the first of equals is the lowest
  for (int i = 0; i < p.K; ++i) {
    Key best = key[0];
    int at = 0;
#pragma unroll
    for (int j = 1; j < PER; ++j)
      if (key[j] > best) {
        best = key[j];
        at = j;
      }
    const Key all = max_lanes<LANES>(best);
    const uint64_t have = __ballot(best == all) >> (sub * LANES);
    const bool mine = __builtin_ctzll(have) == lane;
    if (mine) {
      const bool some = all > (Key)kLowest && wrong == 0.f;
      s_chosen[sub][i] = some ? e0 + at : -1;
#pragma unroll
      for (int j = 0; j < PER; ++j)
        if (j == at) key[j] = kLowest;
    }
  }
  __syncthreads();

  constexpr int TIMES = LANES >= GSQ_MAX_TOP_K ? 1 : GSQ_MAX_TOP_K / LANES;
  double w[TIMES], sum = 0.0;
#pragma unroll
  for (int n = 0; n < TIMES; ++n) {
    const int i = lane + n * LANES, e = i < p.K ? s_chosen[sub][i] : -1;
    w[n] = 0.0;
    if (e >= 0) {
      const double x = s_logit[sub][e];
      w[n] = p.sigmoid ? 1.0 / (1.0 + exp(-x)) : exp(x - (double)top);
    }
    sum += w[n];
  }
  if (p.renormalise) total = sum_lanes<LANES>(sum);
  // the share first: scale / total would overflow where a bias chooses experts whose scores are subnormal
  const double by = wrong != 0.f ? (double)__builtin_nanf("") : total > 0.0 ? (double)p.scale : 0.0;
  if (!(total > 0.0)) total = 1.0;
#pragma unroll
  for (int n = 0; n < TIMES; ++n) {
    const int i = lane + n * LANES;
    if (live && i < p.K) {
      p.experts[token * p.K + i] = s_chosen[sub][i];
      p.weights[token * p.K + i] = (float)(w[n] / total * by);
    }
  }
}

// The gradient of the logits.  A chosen expert j has g_j = scale dw_j.  With D the weighted mean or sum below:
//   softmax, renormalised: p = softmax over the chosen, dl_j = p_j (g_j - D), D = sum_i g_i p_i, no others
//   softmax: dl_e = s_e (sum of e's g) - s_e D, D = sum_i g_i s_i, over all experts
//   sigmoid, renormalised: p = s_j / sum_i s_i, dl_j = p_j (g_j - D) (1 - s_j), D = sum_i g_i p_i, no others
//   sigmoid: dl_j = g_j s_j (1 - s_j), no others
// p is formed from exponentials relative to the chosen experts' largest, so that small scores keep their digits.
template <int LANES, int PER>
__global__ __launch_bounds__(64) void k_route_grad(RouteArgs p) {
  constexpr int TOKENS = 64 / LANES, MOST = LANES * PER;
  constexpr int TIMES = LANES >= GSQ_MAX_TOP_K ? 1 : GSQ_MAX_TOP_K / LANES;
  __shared__ float s_logit[TOKENS][MOST];
  __shared__ int s_chosen[TOKENS][GSQ_MAX_TOP_K];
  __shared__ float s_part[TOKENS][GSQ_MAX_TOP_K];
  const int tid = threadIdx.x, lane = tid % LANES, sub = tid / LANES, e0 = lane * PER;
  const int64_t token = (int64_t)blockIdx.x * TOKENS + sub, row = min(token, p.tokens - 1);
  float l[PER];
  load_logits<PER>(p, row, e0, l);
  int id[TIMES];
  float g[TIMES];
#pragma unroll
  for (int n = 0; n < TIMES; ++n) {
    const int i = lane + n * LANES;
    id[n] = i < p.K ? p.experts[row * p.K + i] : -1;
    if (id[n] >= p.E) id[n] = -1;
    g[n] = id[n] >= 0 ? p.dweights[row * p.K + i] * p.scale : 0.f;
  }
  float top = kLowest;
#pragma unroll
  for (int j = 0; j < PER; ++j) {
    s_logit[sub][e0 + j] = l[j];
    top = fmaxf(top, l[j]);
  }
  __syncthreads();

  const bool dense = !p.sigmoid && !p.renormalise;
  float x[TIMES], s[TIMES], part[TIMES], D = 0.f;
  float chosen_top = kLowest;
#pragma unroll
  for (int n = 0; n < TIMES; ++n) {
    x[n] = id[n] >= 0 ? s_logit[sub][id[n]] : kLowest;
    chosen_top = fmaxf(chosen_top, p.sigmoid ? fminf(x[n], 0.f) : x[n]);
  }
  float inv = 0.f;
  if (dense) {
    top = max_lanes<LANES>(top);
    if (top == kLowest) top = 0.f;
    float sum = 0.f;
#pragma unroll
    for (int j = 0; j < PER; ++j) sum += expf(l[j] - top);
    sum = sum_lanes<LANES>(sum);
    inv = sum != 0.f ? 1.f / sum : 0.f;
  } else {
    chosen_top = max_lanes<LANES>(chosen_top);
    if (chosen_top == kLowest) chosen_top = 0.f;
  }
  float sum = 0.f;
#pragma unroll
  for (int n = 0; n < TIMES; ++n) {
    if (dense) {
      s[n] = expf(x[n] - top) * inv;
    } else if (!p.sigmoid) {
      s[n] = expf(x[n] - chosen_top);
    } else {                                   // e^min(x, 0) / (1 + e^-|x|), for the sums taken by e^chosen_top
      s[n] = expf(fminf(x[n], 0.f) - (p.renormalise ? chosen_top : 0.f)) / (1.f + expf(-fabsf(x[n])));
    }
    if (id[n] < 0) s[n] = 0.f;
    sum += s[n];
  }
  if (p.renormalise) {
    sum = sum_lanes<LANES>(sum);
    inv = sum != 0.f ? 1.f / sum : 0.f;
#pragma unroll
    for (int n = 0; n < TIMES; ++n) s[n] *= inv;
  }
#pragma unroll
  for (int n = 0; n < TIMES; ++n) D += g[n] * s[n];
  D = sum_lanes<LANES>(D);
#pragma unroll
  for (int n = 0; n < TIMES; ++n) {
    part[n] = s[n] * (p.renormalise ? g[n] - D : g[n]);
    if (p.sigmoid) {                           // 1 - s = e^min(-x, 0) / (1 + e^-|x|), without a difference
      part[n] *= expf(fminf(-x[n], 0.f)) / (1.f + expf(-fabsf(x[n])));
    }
    const int i = lane + n * LANES;
    if (i < GSQ_MAX_TOP_K) {
      s_chosen[sub][i] = id[n];
      s_part[sub][i] = id[n] >= 0 ? part[n] : 0.f;
    }
  }
  __syncthreads();

  float d[PER];
#pragma unroll
  for (int j = 0; j < PER; ++j) d[j] = dense ? -D * (expf(l[j] - top) * inv) : l[j] != l[j] ? l[j] : 0.f;
  for (int i = 0; i < p.K; ++i) {
    const int at = s_chosen[sub][i] - e0;
    const float v = s_part[sub][i];
#pragma unroll
    for (int j = 0; j < PER; ++j) d[j] += at == j ? v : 0.f;
  }
  if (token >= p.tokens) return;
  if (p.dtype == GSQ_DT_BF16)
    store_gradient_as(static_cast<__bf16*>(p.dlogits) + token * p.E, p.E, e0, d);
  else if (p.dtype == GSQ_DT_FP16)
    store_gradient_as(static_cast<_Float16*>(p.dlogits) + token * p.E, p.E, e0, d);
  else
    store_gradient_as(static_cast<float*>(p.dlogits) + token * p.E, p.E, e0, d);
}

template <int LANES, int PER>
struct Shape {
  static constexpr int kLanes = LANES, kPer = PER;
};

// Sixteen lanes to a token where there are many, four tokens to a wavefront: the choices then cost least (16384 tokens of
// 256 experts with their order 23.5 us, 27.4 by all 64 lanes).  All 64 for few tokens, whose latency is that of one (64
// tokens of 256 grouped experts with a bias 7.5 us, 17.7 by 16), where more than 128 experts have groups and 64-bit keys
// to look at (16384 of 256 42.6, 49.8 by 16), and beyond 256 experts, which 16 lanes would not hold.
template <class F>
hipError_t with_shape(int64_t tokens, int E, int groups, F f) {
  if (tokens > 2048 && E <= (groups > 1 ? 128 : 256)) {
    if (E <= 64) return f(Shape<16, 4>{});
    return E <= 128 ? f(Shape<16, 8>{}) : f(Shape<16, 16>{});
  }
  if (E <= 64) return f(Shape<64, 1>{});
  if (E <= 128) return f(Shape<64, 2>{});
  if (E <= 256) return f(Shape<64, 4>{});
  return E <= 512 ? f(Shape<64, 8>{}) : f(Shape<64, 16>{});
}

RouteArgs route_args(const gsq_routing& r, const void* logits) {
  RouteArgs p{};
  p.logits = logits;
  p.tokens = r.tokens;
  p.E = r.experts;
  p.K = r.top_k;
  p.groups = r.groups;
  p.top_groups = r.top_groups;
  p.group_size = r.experts / r.groups;
  p.group_inv = ((1u << 20) + p.group_size - 1) / p.group_size;   // exact for e, group_size <= 1024
  p.sigmoid = r.score == GSQ_SCORE_SIGMOID;
  p.top2 = r.group_score == GSQ_GROUP_TOP2;
  p.renormalise = r.renormalise != 0;
  p.scale = r.scale;
  p.dtype = r.dtype;
  return p;
}

// ------------------------------------------------------------------ the order of rows
// Lanes whose ids (of `bits` bits) are this lane's own, among those that have one.
__device__ __forceinline__ uint64_t same_ids(int id, bool some, int bits) {
  uint64_t same = __ballot(some);
  for (int b = 0; b < bits; ++b) {
    const bool one = id >> b & 1;
    const uint64_t ones = __ballot(one);
    same &= one ? ones : ~ones;
  }
  return same;
}

// A wavefront's part of the ids, 64 at a time, counted in a histogram of its own; each id's number among the equal ones
// before it goes to `slots`, or stays in registers with the id where the part is short.
constexpr int kIdsAhead = 4;                // batches whose ids are asked for together
struct HeldIds {
  int id[kIdsAhead], number[kIdsAhead];     // id: -1 of no group
};
__device__ __forceinline__ bool ids_fit(int64_t first, int64_t last) { return last - first <= 64 * kIdsAhead; }

__device__ __forceinline__ void count_ids(const int32_t* ids, int64_t first, int64_t last, int groups, int bits,
                                          uint32_t* hist, int32_t* slots, HeldIds& held) {
  const int lane = threadIdx.x & 63;
  const uint64_t below = ((uint64_t)1 << lane) - 1;
  const bool keep = ids_fit(first, last);
  for (int64_t at = first; at < last; at += 64 * kIdsAhead) {
#pragma unroll
    for (int u = 0; u < kIdsAhead; ++u) {
      const int64_t i = at + u * 64 + lane;
      held.id[u] = i < last ? ids[i] : -1;
    }
#pragma unroll
    for (int u = 0; u < kIdsAhead; ++u) {
      const int64_t i = at + u * 64 + lane;
      if (at + u * 64 >= last) break;
      const bool some = held.id[u] >= 0 && held.id[u] < groups;
      if (!some) held.id[u] = -1;
      const uint64_t same = same_ids(held.id[u], some, bits);
      if (some) {
        const uint32_t before = hist[held.id[u]];
        __builtin_amdgcn_wave_barrier();
        if ((same & below) == 0) hist[held.id[u]] = before + __popcll(same);
        held.number[u] = (int)(before + __popcll(same & below));
        if (!keep) slots[i] = held.number[u];
      }
      __builtin_amdgcn_wave_barrier();
    }
  }
}

// f(index, id, number) for the ids that count_ids has counted, id -1 for those of no group.
template <class F>
__device__ __forceinline__ void each_id(const int32_t* ids, int64_t first, int64_t last, int groups, const int32_t* slots,
                                        const HeldIds& held, F f) {
  const int lane = threadIdx.x & 63;
  if (ids_fit(first, last)) {
#pragma unroll
    for (int u = 0; u < kIdsAhead; ++u)
      if (first + u * 64 + lane < last) f(first + u * 64 + lane, held.id[u], held.number[u]);
    return;
  }
  for (int64_t i = first + lane; i < last; i += 64) {
    const int id = ids[i];
    const bool some = id >= 0 && id < groups;
    f(i, some ? id : -1, some ? slots[i] : 0);
  }
}

// hist[w][g] of all wavefronts becomes the count of the wavefronts before; total(g, n) takes the sum.
template <class Total>
__device__ __forceinline__ void sum_over_waves(uint32_t* hist, int groups, int waves, Total total) {
  for (int g = threadIdx.x; g < groups; g += blockDim.x) {
    uint32_t n = 0;
    for (int w = 0; w < waves; ++w) {
      const uint32_t mine = hist[w * groups + g];
      hist[w * groups + g] = n;
      n += mine;
    }
    total(g, n);
  }
}

// v[0 .. n - 1] in LDS becomes the sum of those before each; the sum of all is returned.
__device__ __forceinline__ uint32_t sums_before(uint32_t* v, int n) {
  __shared__ uint32_t part[16];
  const int tid = threadIdx.x, lane = tid & 63, each = (n + blockDim.x - 1) / blockDim.x;
  const int lo = min(tid * each, n), hi = min(lo + each, n);
  uint32_t sum = 0;
  for (int k = lo; k < hi; ++k) sum += v[k];
  uint32_t upto = sum;
#pragma unroll
  for (int d = 1; d < 64; d <<= 1) {
    const uint32_t x = __shfl_up(upto, d, 64);
    if (lane >= d) upto += x;
  }
  if (lane == 63) part[tid >> 6] = upto;
  __syncthreads();
  uint32_t before = upto - sum, all = 0;
  for (int w = 0; w < (int)(blockDim.x >> 6); ++w) {
    if (w < tid >> 6) before += part[w];
    all += part[w];
  }
  for (int k = lo; k < hi; ++k) {
    const uint32_t mine = v[k];
    v[k] = before;
    before += mine;
  }
  __syncthreads();
  return all;
}

struct OrderArgs {
  const int32_t* ids;
  int64_t count;
  int64_t* offsets;
  int32_t *slots, *sources;
  int32_t groups, bits, waves;   // waves: that count, of a workgroup
  int64_t chunk;                 // ids of a workgroup
  int32_t chunks;
};

// This wavefront's part of the ids [first, last): whole batches of 64.
__device__ __forceinline__ void wave_part(const OrderArgs& p, int64_t& first, int64_t& last) {
  const int wave = threadIdx.x >> 6;
  const int64_t each = ((last - first + p.waves - 1) / p.waves + 63) / 64 * 64;
  const int64_t end = last;
  first = min(first + wave * each, end);
  last = wave < p.waves ? min(first + each, end) : first;
}

// All of it by one workgroup.
__global__ __launch_bounds__(1024) void k_group_few(OrderArgs p) {
  extern __shared__ uint32_t s_hist[];      // waves x groups, then groups
  uint32_t* base = s_hist + p.waves * p.groups;
  const int wave = threadIdx.x >> 6;
  for (int k = threadIdx.x; k < p.waves * p.groups; k += blockDim.x) s_hist[k] = 0;
  __syncthreads();
  int64_t first = 0, last = p.count;
  wave_part(p, first, last);
  HeldIds held;
  count_ids(p.ids, first, last, p.groups, p.bits, s_hist + wave * p.groups, p.slots, held);
  __syncthreads();
  sum_over_waves(s_hist, p.groups, p.waves, [&](int g, uint32_t n) { base[g] = n; });
  __syncthreads();
  const uint32_t all = sums_before(base, p.groups);
  for (int g = threadIdx.x; g < p.groups; g += blockDim.x) p.offsets[g] = base[g];
  if (threadIdx.x == 0) p.offsets[p.groups] = all;
  each_id(p.ids, first, last, p.groups, p.slots, held, [&](int64_t i, int id, int number) {
    int32_t at = -1;
    if (id >= 0) {
      at = number + (int32_t)(s_hist[wave * p.groups + id] + base[id]);
      p.sources[at] = (int32_t)i;
    }
    p.slots[i] = at;
  });
  for (int64_t k = all + threadIdx.x; k < p.count; k += blockDim.x) p.sources[k] = -1;
}

// In three passes: each id's number within its chunk, and the chunks' counts (in `sources`, chunk after chunk);
// the place of each id; and what stands at each place.
__global__ __launch_bounds__(512) void k_group_count(OrderArgs p) {
  extern __shared__ uint32_t s_hist[];      // waves x groups
  const int wave = threadIdx.x >> 6;
  for (int k = threadIdx.x; k < p.waves * p.groups; k += blockDim.x) s_hist[k] = 0;
  __syncthreads();
  int64_t first = blockIdx.x * p.chunk, last = min(first + p.chunk, p.count);
  wave_part(p, first, last);
  HeldIds held;
  count_ids(p.ids, first, last, p.groups, p.bits, s_hist + wave * p.groups, p.slots, held);
  __syncthreads();
  uint32_t* table = reinterpret_cast<uint32_t*>(p.sources) + (int64_t)blockIdx.x * p.groups;
  sum_over_waves(s_hist, p.groups, p.waves, [&](int g, uint32_t n) { table[g] = n; });
  __syncthreads();
  each_id(p.ids, first, last, p.groups, p.slots, held, [&](int64_t i, int id, int number) {
    if (id >= 0) p.slots[i] = number + (int32_t)s_hist[wave * p.groups + id];
  });
}

__global__ __launch_bounds__(512) void k_group_place(OrderArgs p) {
  extern __shared__ uint32_t s_base[];      // groups, groups, and the shares' parts
  const uint32_t* table = reinterpret_cast<const uint32_t*>(p.sources);
  uint32_t* mine = s_base + p.groups;
  // few groups: several threads to each, with a part of the chunks
  const int shares = max(1, (int)blockDim.x / p.groups);
  uint32_t* part_all = shares > 1 ? mine + p.groups : s_base;
  uint32_t* part_before = shares > 1 ? part_all + shares * p.groups : mine;
  for (int t = threadIdx.x; t < shares * p.groups; t += blockDim.x) {
    const int g = t % p.groups;
    uint32_t all = 0, before = 0;
#pragma unroll 8
    for (int c = t / p.groups; c < p.chunks; c += shares) {
      const uint32_t n = table[(int64_t)c * p.groups + g];
      before += c < (int)blockIdx.x ? n : 0;
      all += n;
    }
    part_all[t] = all;
    part_before[t] = before;
  }
  __syncthreads();
  for (int g = threadIdx.x; g < p.groups; g += blockDim.x) {
    uint32_t all = 0, before = 0;
    for (int t = g; t < shares * p.groups; t += p.groups) {
      all += part_all[t];
      before += part_before[t];
    }
    s_base[g] = all;
    mine[g] = before;
  }
  __syncthreads();
  const uint32_t all = sums_before(s_base, p.groups);
  if (blockIdx.x == 0) {
    for (int g = threadIdx.x; g < p.groups; g += blockDim.x) p.offsets[g] = s_base[g];
    if (threadIdx.x == 0) p.offsets[p.groups] = all;
  }
  const int64_t first = blockIdx.x * p.chunk, last = min(first + p.chunk, p.count);
  for (int64_t i = first + threadIdx.x; i < last; i += blockDim.x) {
    const int id = p.ids[i];
    p.slots[i] = id >= 0 && id < p.groups ? p.slots[i] + (int32_t)(s_base[id] + mine[id]) : -1;
  }
}

__global__ __launch_bounds__(256) void k_group_sources(OrderArgs p) {
  const int64_t all = p.offsets[p.groups];
  for (int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x; i < p.count; i += (int64_t)gridDim.x * 256) {
    const int32_t at = p.slots[i];
    if (at >= 0) p.sources[at] = (int32_t)i;
    if (i >= all) p.sources[i] = -1;
  }
}

__global__ void k_no_rows(OrderArgs p) {
  for (int g = threadIdx.x; g <= p.groups; g += blockDim.x) p.offsets[g] = 0;
}

}  // namespace

hipError_t launch_route(const gsq_routing& r, const void* logits, const float* bias, int32_t* experts, float* weights,
                        hipStream_t s) {
  if (r.tokens == 0) return hipSuccess;
  RouteArgs p = route_args(r, logits);
  p.bias = bias;
  p.experts = experts;
  p.weights = weights;
  return with_shape(r.tokens, r.experts, r.groups, [&](auto shape) {
    using S = decltype(shape);
    constexpr int LANES = S::kLanes, PER = S::kPer, TOKENS = 64 / LANES;
    const int64_t blocks = tiles_of(r.tokens, TOKENS);
    const size_t lds = r.groups > 1 ? (size_t)TOKENS * (LANES * PER + LANES * PER / 16) * sizeof(double) : 0;
    while (2 << p.group_share <= LANES / r.groups) ++p.group_share;
    if (!fits_launch(blocks, 64)) return hipErrorInvalidConfiguration;
    if (bias)
      k_route<double, LANES, PER><<<(unsigned)blocks, 64, lds, s>>>(p);
    else
      k_route<float, LANES, PER><<<(unsigned)blocks, 64, lds, s>>>(p);
    return hipGetLastError();
  });
}

hipError_t launch_route_grad(const gsq_routing& r, const void* logits, const int32_t* experts, const float* dweights,
                             void* dlogits, hipStream_t s) {
  if (r.tokens == 0) return hipSuccess;
  RouteArgs p = route_args(r, logits);
  p.experts = const_cast<int32_t*>(experts);
  p.dweights = dweights;
  p.dlogits = dlogits;
  return with_shape(r.tokens, r.experts, 1, [&](auto shape) {
    using S = decltype(shape);
    const int64_t blocks = tiles_of(r.tokens, 64 / S::kLanes);
    if (!fits_launch(blocks, 64)) return hipErrorInvalidConfiguration;
    k_route_grad<S::kLanes, S::kPer><<<(unsigned)blocks, 64, 0, s>>>(p);
    return hipGetLastError();
  });
}

hipError_t launch_group_rows(const int32_t* ids, int64_t count, int groups, int64_t* offsets, int32_t* slots,
                             int32_t* sources, hipStream_t s) {
  OrderArgs p{ids, count, offsets, slots, sources, groups, 0, 0, 0, 0};
  while (1 << p.bits < groups) ++p.bits;
  if (count == 0) {
    k_no_rows<<<1, 256, 0, s>>>(p);
    return hipGetLastError();
  }
  const OrderPlan plan = plan_order(count, groups);
  p.waves = plan.waves;
  p.chunk = plan.chunk;
  p.chunks = plan.chunks;
  if (plan.chunks == 1) {
    k_group_few<<<1, plan.threads, ((size_t)p.waves + 1) * groups * 4, s>>>(p);
    return hipGetLastError();
  }
  k_group_count<<<p.chunks, plan.threads, (size_t)p.waves * groups * 4, s>>>(p);
  hipError_t e = hipGetLastError();
  if (e != hipSuccess) return e;
  k_group_place<<<p.chunks, plan.threads, (size_t)(2 * groups + (groups < plan.threads ? 2 * plan.threads : 0)) * 4, s>>>(p);
  if ((e = hipGetLastError()) != hipSuccess) return e;
  k_group_sources<<<(unsigned)std::min<int64_t>(tiles_of(count, 256), 16384), 256, 0, s>>>(p);
  return hipGetLastError();
}

}  // namespace gsq
