/*
 * iwp_loss.h - C ABI of the losses whose gradients the pruned all-reduce step of iwp.h takes: the output head of a
 *              model with its softmax cross entropy, the same head against a teacher's top logits, and the balance
 *              loss of a router over experts.  Same library (libiwp.so), same status codes.
 *
 * Conventions as in iwp.h: int status, nothing throws or aborts, pointers are DEVICE pointers unless named *_host,
 * the caller owns every buffer.  No call here allocates, synchronises or keeps anything between calls; all scratch is
 * the caller's `workspace` (one per stream: calls that share a workspace must not overlap on the GPU).  What outlives a
 * call is in the IWP_LOSS_STATE bytes of `state`, or of the workspace's beginning if `state` is NULL: a status word
 * that kernels set and iwp_loss_status() reads, and counters.  They are made ready by iwp_loss_reset() once; the rest of
 * a workspace needs no preparation, so with a `state` of its own a workspace may be exchanged for another at any time.
 */
#ifndef IWP_LOSS_H_
#define IWP_LOSS_H_

#include <stdint.h>

#include "iwp.h"

#ifdef __cplusplus
extern "C" {
#endif

enum { IWP_F32 = 0, IWP_BF16 = 1, IWP_F16 = 2 }; /* element types */
enum { IWP_LOSS_STATE = 256 };

/* Zeroes a state (or the one at a workspace's beginning), in stream order.  Errors: IWP_ERR_INVALID (NULL), IWP_ERR_CUDA. */
int iwp_loss_reset(void* state, void* cuda_stream);

/* Copies a state's (or a workspace's) status word to *status_host behind everything enqueued on cuda_stream and waits
 * for that stream: IWP_OK; IWP_ERR_INVALID (a target or teacher id outside the vocabulary was met); IWP_ERR_TIMEOUT
 * (a bounded device-side wait gave up; results are undefined).  Errors: IWP_ERR_INVALID (NULL), IWP_ERR_CUDA. */
int iwp_loss_status(const void* state, int32_t* status_host, void* cuda_stream);

/* ---- output head with its loss ---------------------------------------------------------------------
 *
 * logits z[t][v] = <hidden[t], weight[v]> exist tile by tile in tensor memory; forward passes keep none of them.  While
 * the gradients of a piece of the vocabulary are formed, its probabilities are held in 16 bits: at most piece_bytes, by
 * default up to max(1 GiB, 4 V D bytes), which for many vocabularies is all of them.
 * Row t has sparse targets (i_k, q_k), sum of q = 1, or none.  With tau = temperature (1 for the cross entropy)
 *   lse[t]  = log sum_v exp(z[t][v] / tau)
 *   rows[t] = tau^2 * sum_k q_k (log q_k - z[t][i_k] / tau + lse[t])      (a row without targets: 0)
 *   loss    = sum_t rows[t], divided by the number of rows with targets if `mean` (0 if there is none)
 *   dz[t][v] = g_t * tau * (exp(z[t][v] / tau - lse[t]) - q of v),  g_t = dloss_rows[t] * dloss * scale (/ number)
 *   dhidden = dz weight,  dweight = dz^T hidden                            (rows without targets give nothing,
 *                                                          whatever their hidden states hold)
 * Cross entropy (targets != NULL): q = 1 at targets[t]; targets[t] == ignore_index: no target.  Distillation
 * (targets == NULL): q = softmax over the row's top_k teacher logits / tau; an id below 0 is padding and takes no
 * part, a logit of -inf has q = 0; nothing but those: no target.  A target or id at or above vocab (or a negative
 * target that is not ignore_index) sets the status word to IWP_ERR_INVALID, makes the row's loss NaN and gives no
 * gradient; the row still counts as one with a target.
 * Products are of the operands' 16-bit type with fp32 accumulation; statistics and losses are fp32.
 * The gradient's factors exp(..) - q are rounded to the operands' type, as the tensor cores take no wider one.  Where
 * nothing is subtracted, exp(..) may have been held in a 16-bit code before: off by at most 2^-12 of itself (bf16
 * operands) or 1.7e-4 (fp16), and nothing below 2^-40 (2^-24) of the largest of the row's 32 to 128 columns around it.
 * Where q is subtracted, exp(..) is fp32: a student close to its teacher keeps the precision of one rounding.
 * A row's dhidden depends on no other row's dloss_rows, neither in its precision nor by an infinity or NaN.  With fp16
 * operands and dloss_rows, dweight sums over hidden states multiplied by powers of two of at most 1 and rounded to fp16.
 */
typedef struct iwp_head_args {
  int64_t tokens, vocab, dim;      /* T >= 0, 1 <= V, 1 <= D; each at most 2^31 - 2^16, their products
                                      at most 2^46 */
  const void* hidden;              /* [T][D], row stride hidden_ld elements */
  int64_t hidden_ld;
  const void* weight;              /* [V][D], row stride weight_ld elements */
  int64_t weight_ld;
  const int64_t* targets;          /* [T], or NULL: distillation */
  int64_t ignore_index;
  const void* top_ids;             /* [T][top_k] of int32 or int64 (ids_bytes), row stride top_ids_ld */
  int64_t top_ids_ld;
  const void* top_logits;          /* [T][top_k] of top_type, row stride top_logits_ld */
  int64_t top_logits_ld;
  float* loss;                     /* 1, or NULL */
  float* rows;                     /* [T], or NULL */
  float* lse;                      /* [T]; read instead of written if have_lse */
  const float* dloss;              /* 1 on the device, or NULL = 1 */
  const float* dloss_rows;         /* [T], or NULL = 1 */
  void* dhidden;                   /* [T][D] of dhidden_type, or NULL */
  int64_t dhidden_ld;
  void* dweight;                   /* [V][D] of dweight_type, or NULL */
  int64_t dweight_ld;
  void* workspace;                 /* 256-byte aligned */
  int64_t workspace_bytes;
  void* state;                     /* IWP_LOSS_STATE bytes, 256-byte aligned, or NULL: the workspace's first */
  int64_t piece_bytes;             /* bound on the probabilities of one piece of the vocabulary; 0 = 1 GiB, or what the
                                      weights and their gradient take (4 V D bytes) where that is more */
  float temperature, scale;
  int32_t dtype;                   /* IWP_BF16 or IWP_F16: hidden and weight */
  int32_t top_k, ids_bytes, top_type; /* 1 <= top_k <= 1024 */
  int32_t dhidden_type, dweight_type; /* dtype or IWP_F32 */
  int32_t mean;                    /* 1 = mean over rows with targets, 0 = sum */
                                   /* (outputs overlap neither inputs nor one another) */
  int32_t accumulate;              /* 1 = the gradients are added to what dhidden and dweight hold */
  int32_t have_lse;                /* 1 = lse is given: no forward pass, loss and rows are not written */
} iwp_head_args;

/* Bytes of workspace a call with these arguments needs (pointers matter only by being NULL or not, and by their
 * alignment: operands whose rows do not start at multiples of 16 bytes are first copied to rows that do): the
 * statistics, T D elements where dweight is asked for, the probabilities of a piece, and 78 MB or 4 T D bytes for
 * partial sums where dhidden is.  It does not shrink when tokens grow.  -1 = invalid arguments. */
int64_t iwp_head_workspace(const iwp_head_args* args);

/* Loss, and the gradients that are not NULL.  Asynchronous on cuda_stream.  Errors: IWP_ERR_INVALID (sizes, NULL,
 * types, strides), IWP_ERR_CAPACITY (workspace too small), IWP_ERR_CUDA. */
int iwp_head_loss(const iwp_head_args* args, void* cuda_stream);

/* ---- balance loss of a router ----------------------------------------------------------------------
 *
 * n = number of tokens with mask != 0 (all, if mask is NULL); p_t = softmax(logits[t])
 *   counts[e] = number of pairs (t, j) with mask[t] and ids[t][j] == e        (ids outside [0, E) are dropped)
 *   f_e = counts[e] / (n * top_k),  mean_prob[e] = sum_t mask[t] p_t[e] / n
 *   loss = coef * E * sum_e f_e mean_prob[e]
 *   dlogits[t][e] = scale * dloss * coef * E / n * mask[t] * p_t[e] * (f_e - sum_j f_j p_t[j])
 * n = 0: all results 0.  Logits of -inf have p = 0; a row of nothing else contributes nothing.
 * Sums are of fixed order: equal inputs give equal bits.
 */
typedef struct iwp_balance_args {
  int64_t tokens;                  /* T >= 0 */
  const void* logits;              /* [T][E] of type, row stride logits_ld */
  int64_t logits_ld;
  const void* ids;                 /* [T][top_k] of int32 or int64 (ids_bytes), row stride ids_ld */
  int64_t ids_ld;
  const uint8_t* mask;             /* [T], or NULL */
  const float* dloss;              /* 1 on the device, or NULL = 1 */
  float* loss;                     /* 1, or NULL */
  int32_t* counts;                 /* [E] */
  float* mean_prob;                /* [E], or NULL */
  void* dlogits;                   /* [T][E] of type, or NULL */
  int64_t dlogits_ld;
  void* workspace;                 /* 256-byte aligned */
  int64_t workspace_bytes;
  void* state;                     /* as in iwp_head_args */
  float coef, scale;
  int32_t experts, top_k;          /* 1 <= E <= 1024, 1 <= top_k <= E */
  int32_t type, ids_bytes;
} iwp_balance_args;

int64_t iwp_balance_workspace(const iwp_balance_args* args); /* -1 = invalid arguments */
int iwp_balance_loss(const iwp_balance_args* args, void* cuda_stream); /* errors as iwp_head_loss() */

#ifdef __cplusplus
}
#endif
#endif /* IWP_LOSS_H_ */
