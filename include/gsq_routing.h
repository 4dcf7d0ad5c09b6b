/*
 * gsq_routing.h -- rows to the routed experts and back, in the same library as gsq.h.
 *
 * What stands around the products of gsq_products.h when the layers of a batch are routed experts: each
 * token's experts and weights from its logits (gsq_route), the order in which the rows of all experts come
 * together (gsq_group_rows, whose offsets the products take), the tokens copied into that order
 * (gsq_dispatch_rows) and the experts' rows summed back (gsq_combine_rows), with their gradients.
 *
 * Stream, device pointers, status codes and gsq_last_error() are as gsq.h says, addresses, overlapping calls
 * and reproducibility as gsq_products.h does: dense row-major arrays, aligned to their elements; nothing is
 * allocated, synchronised or kept, and the host reads no device memory, so that every call can be captured.
 */
#ifndef GSQ_ROUTING_H
#define GSQ_ROUTING_H

#include "gsq_products.h"

#ifdef __cplusplus
extern "C" {
#endif

enum { GSQ_SCORE_SOFTMAX = 0, GSQ_SCORE_SIGMOID = 1 };   /* of a token's logits       */
enum { GSQ_GROUP_MAX = 0, GSQ_GROUP_TOP2 = 1 };          /* what a group is chosen by */
#define GSQ_MAX_EXPERTS 1024
#define GSQ_MAX_TOP_K 32
#define GSQ_MAX_EXPERT_GROUPS 64
#define GSQ_MAX_ROW_GROUPS 4096

typedef struct {
  int64_t tokens;          /* T (>= 0, <= 2^25)                                                    */
  int32_t experts;         /* E (1 .. GSQ_MAX_EXPERTS)                                             */
  int32_t top_k;           /* K experts of a token (1 .. GSQ_MAX_TOP_K, <= top_groups E / groups)  */
  int32_t groups;          /* of E / groups consecutive experts each (1: none; <= 64, divides E)   */
  int32_t top_groups;      /* groups that a token's experts come from (1 .. groups)                */
  int32_t score;           /* GSQ_SCORE_*                                                          */
  int32_t group_score;     /* GSQ_GROUP_*                                                          */
  int32_t renormalise;     /* != 0: the weights of a token's experts add up to scale               */
  float scale;             /* of the weights (finite)                                              */
  int32_t dtype;           /* of the logits and their gradient: GSQ_DT_*                           */
} gsq_routing;

/* The experts of each token.  logits: T x E, bias: fp32 E or NULL, experts: int32 T x K, weights: fp32 T x K.
 *
 * s = softmax or sigmoid of the token's logits.  An expert's key is s + bias (64 bits); without a bias experts
 * are ordered by their logits.  With groups > 1 a group counts its largest s + bias, or the sum of its two
 * largest (GSQ_GROUP_TOP2; one, where it has no second), and only experts of the top_groups best groups are
 * left.  The K experts with the largest keys follow in that order; ties go to the lowest index.  The bias
 * chooses only: weights = scale s, or scale s / (sum of s of the chosen); where that sum is zero, zero.
 *
 * A logit of -infinity, and a key that is -infinity or NaN, means that the expert is not there.  A token with
 * fewer than K experts (a row of padding has none) has experts -1 with weight 0 in the places left.  A token
 * with a logit that is NaN, or +infinity under softmax, has experts -1 and weights NaN. */
gsq_status gsq_route(const gsq_routing* r, const void* logits, const float* bias, int32_t* experts,
                     float* weights, hipStream_t stream);

/* The gradient of the logits from dweights (fp32 T x K), the choice being constant: experts as gsq_route wrote
 * them (others than 0 .. E - 1 have none), dlogits: T x E in dtype.  groups, top_groups and group_score are
 * checked, not used. */
gsq_status gsq_route_grad(const gsq_routing* r, const void* logits, const int32_t* experts,
                          const float* dweights, void* dlogits, hipStream_t stream);

/* The order that brings equal ids together: a stable sort of ids[0 .. count - 1] by group (0 .. groups - 1;
 * others belong to none and are left out).  offsets: int64 groups + 1, as the products take them, slots: int32
 * count, the place of each id or -1, sources: int32 count, the index that stands at each place and -1 behind
 * the last.  count <= 2^30, groups <= GSQ_MAX_ROW_GROUPS.  For gsq_route's experts, count = T K, and place p
 * is a copy of token sources[p] / K.  The outputs must not overlap (sources is also used on the way). */
gsq_status gsq_group_rows(const int32_t* ids, int64_t count, int32_t groups, int64_t* offsets, int32_t* slots,
                          int32_t* sources, hipStream_t stream);

typedef struct {
  int64_t tokens;          /* T (>= 0, <= 2^29)                                            */
  int64_t rows;            /* R: rows in the experts' order (>= 0, <= 2^29)                */
  int32_t copies;          /* K: slots of a token (1 .. 1024)                              */
  int32_t cols;            /* C: columns of a row (1 .. 2^21)                              */
  int32_t dtype;           /* of tokens and rows: GSQ_DT_*                                 */
} gsq_exchange;

/* out[slots[t, k]] = x[t].  x: T x C, slots: int32 T x K, out: R x C.  Slots outside 0 .. R - 1 name no row; rows
 * that no slot names are left as they were.  Slots of different tokens have to be distinct: each value of a row
 * that several name is that of one of them, not always the same one. */
gsq_status gsq_dispatch_rows(const gsq_exchange* g, const void* x, const int32_t* slots, void* out,
                             hipStream_t stream);

/* out[t] = sum_k weights[t, k] rows[slots[t, k]], in fp32 in the order of k, rounded once.  rows: R x C, weights:
 * fp32 T x K or NULL (ones), out: T x C.  A slot that names no row counts as a row of zeros (a weight that is
 * not finite shows as NaN). */
gsq_status gsq_combine_rows(const gsq_exchange* g, const void* rows, const int32_t* slots, const float* weights,
                            void* out, hipStream_t stream);

/* Its gradients from dout (T x C): drows[slots[t, k]] = weights[t, k] dout[t] (R x C in dtype; rows that no slot
 * names are left as they were; slots have to be distinct, as above, those of one token too) and dweights[t, k] =
 * sum_c dout[t, c] rows[slots[t, k], c] (fp32 T x K; 0 for a slot that names no row). */
gsq_status gsq_combine_rows_grad(const gsq_exchange* g, const void* dout, const void* rows, const int32_t* slots,
                                 const float* weights, void* drows, float* dweights, hipStream_t stream);

#ifdef __cplusplus
}
#endif

#endif /* GSQ_ROUTING_H */
