/*
 * iwp_clip.h - C ABI of norms and clipping of gradient tensors, as they are on their way into the pruned all-reduce step of
 *              iwp.h: many tensors of mixed types, in groups (a worker each, say) with a norm of their own, clipped where
 *              they are or on the way into a worker's fp32 segment.  Same library (libiwp.so), same status codes.
 *
 * Conventions as in iwp_loss.h: int status, nothing throws or aborts, the caller owns every buffer, no call allocates or
 * synchronises.  Where the tensors are is laid out once, by iwp_clip_table() in host memory; the caller copies that table to
 * the device and hands it to every call.  `state` is as in iwp_loss.h (iwp_loss_reset() makes it ready).  Equal inputs in
 * equal layouts (types, strides, alignment) give equal bits.
 */
#ifndef IWP_CLIP_H_
#define IWP_CLIP_H_

#include <stdint.h>

#include "iwp_loss.h"

#ifdef __cplusplus
extern "C" {
#endif

typedef struct iwp_clip_tensor {
  const void* in;                  /* device: [rows][cols] of in_type, row stride in_ld elements */
  void* out;                       /* device: [rows][cols] of out_type, row stride out_ld; may be `in` itself with the same
                                      type and stride; otherwise it overlaps no input and no other output.  NULL: norms only */
  int64_t rows, cols, in_ld, out_ld; /* rows, cols >= 0; rows cols <= 2^46 */
  int32_t group, in_type, out_type;
} iwp_clip_tensor;

/* Sizes of the table of `n` tensors in `groups` groups; host only. */
typedef struct iwp_clip_sizes {
  int64_t table_bytes;             /* of the table, 16-byte aligned on the device */
  int64_t workspace_bytes;         /* of every call's workspace */
  int64_t parts, warps;            /* for iwp_clip_args */
  int64_t range;                   /* work of a warp, for information: iwp_clip_table() shares the work out again */
} iwp_clip_sizes;

/* Errors: IWP_ERR_INVALID (NULL, sizes, types, alignment below the type's size, groups outside [0, groups), more than 2^25
 * rows), IWP_ERR_OOM (host memory). */
int iwp_clip_layout(const iwp_clip_tensor* tensors_host, int64_t n, int32_t groups, iwp_clip_sizes* sizes_host);
int iwp_clip_table(const iwp_clip_tensor* tensors_host, int64_t n, int32_t groups, void* table_host, int64_t table_bytes);

/* For every group g, over all its tensors' elements x:
 *   squares[g] = sum x^2                        (64 bits; have_squares: read instead, e.g. added up over ranks)
 *   norms[g]   = |scale| sqrt(squares[g])
 *   factors[g] = scale * (norms[g] > max_norm ? max_norm / norms[g] : 1)
 *   out        = factors[g] * x in fp32, rounded again to an output of 16 bits   (`write`; the factor as fp32 has it)
 * A group without elements has norm 0.  A group whose sum is not finite (a NaN or an infinity in a gradient) has factor
 * `scale`, or, with drop_nonfinite, 0, and its outputs are then 0 whatever the elements are.  A factor of exactly 1 leaves tensors that are clipped where
 * they are untouched. */
typedef struct iwp_clip_args {
  const void* table;               /* device */
  int64_t parts, warps;            /* of iwp_clip_layout() */
  double* squares;                 /* [groups] */
  float* norms;                    /* [groups] */
  float* factors;                  /* [groups]; may be NULL without `write` */
  void* workspace;                 /* 256-byte aligned */
  int64_t workspace_bytes;
  void* state;                     /* IWP_LOSS_STATE bytes, 256-byte aligned */
  double max_norm, scale;          /* max_norm >= 0 (infinity: no clipping); scale finite, not 0 */
  int32_t groups;                  /* 1 <= groups <= 2^20 */
  int32_t write, have_squares, drop_nonfinite;
} iwp_clip_args;

int iwp_clip(const iwp_clip_args* args, void* cuda_stream); /* Errors: IWP_ERR_INVALID, IWP_ERR_CAPACITY (workspace), IWP_ERR_CUDA. */

#ifdef __cplusplus
}
#endif
#endif /* IWP_CLIP_H_ */
