/*
 * iwp_route.h - C ABI of a router over experts: the choice of experts with its weights and their gradient, and the
 *               exchange of rows between tokens and experts.  It goes with the balance loss of iwp_loss.h, whose ids
 *               and counts these are.  Same library (libiwp.so), same status codes.
 *
 * Conventions as in iwp_loss.h: int status, nothing throws or aborts, pointers are DEVICE pointers, the caller owns every
 * buffer, no call allocates or synchronises.  What outlives a call is in the IWP_ROUTE_STATE bytes of `state`: counters
 * that iwp_route_reset() zeroes once and every call leaves at zero (one state per stream: calls that share one must not
 * overlap on the GPU).  Outputs overlap neither inputs nor one another.  Equal inputs in equal layouts (types, strides, alignment) give equal bits.
 */
#ifndef IWP_ROUTE_H_
#define IWP_ROUTE_H_

#include <stdint.h>

#include "iwp_loss.h"

#ifdef __cplusplus
extern "C" {
#endif

enum { IWP_ROUTE_STATE = 256 + 4096 };
enum { IWP_SOFTMAX = 0, IWP_SIGMOID = 1 }; /* scores */

/* Zeroes a state, in stream order.  Errors: IWP_ERR_INVALID (NULL), IWP_ERR_CUDA. */
int iwp_route_reset(void* state, void* cuda_stream);

/* ---- routing ------------------------------------------------------------------------------------------
 *
 * s[t][e] = softmax over e of logits[t], or sigmoid(logits[t][e])
 * c[t][e] = s[t][e] + bias[e]: the choice goes by c, the weights by s.  Without a bias the experts are ordered by their
 *   logits, which order the scores.  Where rounding could change the choice it is made again in 64 bits.
 * With groups > 1, group q has the experts [q E / groups, (q + 1) E / groups); it is scored by the sum of its group_top
 *   (1 or 2) largest c, and only the top_groups best groups (ties: the lower one) take part in the choice.
 * ids[t] = the top_k experts of the largest c in descending order, ties: the lower expert first
 * p[t][j] = s[t][ids[t][j]], divided by the sum of the row's chosen s if `renormalize`
 * weights[t][j] = weight_scale * p[t][j];  counts[e] = number of pairs (t, j) with ids[t][j] == e
 * An expert whose logit or bias is -inf (or whose bias is NaN) is not available: not chosen, and no other is in its place,
 * so a row of fewer than top_k available experts ends in ids of -1 with weights 0.  A group with fewer than group_top
 * available experts is scored -inf.  A row with mask[t] == 0 has ids -1 and weights 0; a row that holds a NaN (or, for
 * softmax, +inf) has ids -1 and weights NaN.  A row's ids do not depend on the other rows or on how many there are; its
 * weights may differ in the last places between calls of fewer and of more than 24576 rows, which sum in another order.
 */
typedef struct iwp_route_args {
  int64_t tokens;                  /* 0 <= T <= 2^30, T E <= 2^46 */
  const void* logits;              /* [T][E] of type, row stride logits_ld elements */
  int64_t logits_ld;
  const float* bias;               /* [E], or NULL */
  const uint8_t* mask;             /* [T], or NULL */
  void* ids;                       /* [T][top_k] of int32 or int64 (ids_bytes) */
  float* weights;                  /* [T][top_k] */
  int32_t* counts;                 /* [E], or NULL */
  void* state;                     /* IWP_ROUTE_STATE bytes, 256-byte aligned */
  float weight_scale;              /* finite, not 0 */
  int32_t experts, top_k;          /* 1 <= E <= 1024, 1 <= top_k <= 32 and <= E top_groups / groups */
  int32_t groups, top_groups, group_top; /* 1 <= groups <= 32, divides E; group_top <= E / groups */
  int32_t score, renormalize;
  int32_t type, ids_bytes;
} iwp_route_args;

int iwp_route(const iwp_route_args* args, void* cuda_stream); /* Errors: IWP_ERR_INVALID (sizes, NULL, types, strides), IWP_ERR_CUDA. */

/* The gradient to the logits, for an upstream gradient dweights and the ids and weights of iwp_route():
 *   renormalized: b_j = weights[t][j] sum_i p_i (dweights[t][j] - dweights[t][i]),  p_i = weights[t][i] / weight_scale
 *   else:         b_j = weights[t][j] dweights[t][j]
 *   softmax: dlogits[t][e] = sum of b_j over j with ids[t][j] == e,  less s_e sum_j b_j if not renormalized
 *   sigmoid: dlogits[t][e] = (1 - s_e) (sum of those b_j)
 * ids outside [0, E) take no part and give nothing; a row of nothing else (and, without renormalization, any expert of
 * logit -inf) gets 0. */
typedef struct iwp_route_grad_args {
  int64_t tokens;
  const void* logits;              /* as above; read where the formula has s */
  int64_t logits_ld;
  const void* ids;                 /* [T][top_k], row stride ids_ld */
  int64_t ids_ld;
  const float* weights;            /* [T][top_k], row stride weights_ld */
  int64_t weights_ld;
  const float* dweights;           /* [T][top_k], row stride dweights_ld */
  int64_t dweights_ld;
  void* dlogits;                   /* [T][E] of type */
  int64_t dlogits_ld;
  float weight_scale, scale;       /* the gradient is multiplied by `scale` */
  int32_t experts, top_k;
  int32_t score, renormalize;
  int32_t type, ids_bytes;
  int32_t accumulate;              /* 1 = added to what dlogits holds, e.g. the balance loss's gradient */
} iwp_route_grad_args;

int iwp_route_grad(const iwp_route_grad_args* args, void* cuda_stream);

/* ---- exchange of rows ----------------------------------------------------------------------------------
 *
 * A pair (t, j) belongs to expert ids[t][j]; ids outside [0, E) belong to none.  Sorted by expert, then by token, then by j,
 * the pairs take the slots 0, 1, ...: expert e's are [offsets[e], offsets[e + 1]).
 */
typedef struct iwp_order_args {
  int64_t tokens;                  /* T >= 0, T top_k <= 2^30 */
  const void* ids;                 /* [T][top_k] of int32 or int64 (ids_bytes), row stride ids_ld */
  int64_t ids_ld;
  int32_t* offsets;                /* [E + 1] */
  int32_t* slots;                  /* [T][top_k]: slot of each pair, -1 = none */
  int32_t* rows;                   /* [T top_k]: token of each slot, -1 behind the last one */
  void* workspace;                 /* 256-byte aligned */
  int64_t workspace_bytes;
  int32_t experts, top_k;          /* 1 <= E <= 1024, 1 <= top_k <= 32 */
  int32_t ids_bytes;
} iwp_order_args;

int64_t iwp_order_workspace(const iwp_order_args* args); /* -1 = invalid arguments */
int iwp_order(const iwp_order_args* args, void* cuda_stream); /* also IWP_ERR_CAPACITY (workspace too small) */

/* dispatch:     by_slot_out[slot of (t, j)] = by_token[t];  rows behind offsets[E] are set to zero
 * combine:      by_token_out[t] = sum_j weights[t][j] by_slot[slot of (t, j)], in fp32 and in the order of j, rounded once;
 *               weights NULL: 1 (the gradient of dispatch)
 * combine_grad: by_slot_out[slot of (t, j)] = weights[t][j] by_token[t];  rows behind offsets[E] are set to zero
 *               dweights[t][j] = <by_token[t], by_slot[slot of (t, j)]>, 0 for a pair without a slot
 * Slots outside [0, T top_k) are none.  Rows of slots below offsets[E] that no pair has (of an order that was changed by hand) are
 * left as they are. */
typedef struct iwp_exchange_args {
  int64_t tokens, dim;             /* T top_k <= 2^30, D <= 2^31 - 2^16, T top_k D <= 2^46 */
  const int32_t* slots;            /* [T][top_k], of iwp_order() */
  const int32_t* offsets;          /* [E + 1] */
  const void* by_token;            /* [T][D] of type, row stride by_token_ld */
  int64_t by_token_ld;
  const void* by_slot;             /* [T top_k][D] of type, row stride by_slot_ld */
  int64_t by_slot_ld;
  const float* weights;            /* [T][top_k], row stride weights_ld, or NULL */
  int64_t weights_ld;
  void* by_token_out;              /* [T][D] */
  int64_t by_token_out_ld;
  void* by_slot_out;               /* [T top_k][D]; combine_grad: or NULL */
  int64_t by_slot_out_ld;
  float* dweights;                 /* [T][top_k]; or NULL */
  int32_t experts, top_k;
  int32_t type;
} iwp_exchange_args;

int iwp_dispatch(const iwp_exchange_args* args, void* cuda_stream);
int iwp_combine(const iwp_exchange_args* args, void* cuda_stream);
int iwp_combine_grad(const iwp_exchange_args* args, void* cuda_stream);

#ifdef __cplusplus
}
#endif
#endif /* IWP_ROUTE_H_ */
