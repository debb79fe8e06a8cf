/*
 * nvfp4_finetune -- recovering, and serving, a model whose weights are quantized to NVFP4 (same library and
 * conventions as nvfp4_46.h: device pointers, caller's memory and stream, an nvfp4_status back, nothing enqueued
 * by a call that is refused).
 *
 *   nvfp4_adapters_*   low-rank adapters of many requests at once, beside a projection that they share: the weight stays
 *                      quantized and frozen, adapters hold the correction
 *   nvfp4_distill_*    the divergence of a model's logits from a teacher's top logits, and its gradient
 *
 * Matrices are row-major with a stride in elements from row to row; columns are adjacent.  Infinities and NaN are carried as
 * fp32 arithmetic carries them.  Results do not depend on what else runs and are the same, bit for bit, from call to call.
 * With no tokens (no rows) a call is accepted, and pointers to what has one value or row per token may be NULL.
 */
#ifndef NVFP4_FINETUNE_H
#define NVFP4_FINETUNE_H

#include "../nvfp4_46.h"

#ifdef __cplusplus
extern "C" {
#endif

/* ---- low-rank adapters ----------------------------------------------------------------------------------------
 *
 * Adapter l is the pair A_l [rank][inp], B_l [out][rank] (BF16) and a scale s_l (fp32).  Token t has the adapter
 * l = which[t]; a value outside [0, adapters) means that it has none.  Tokens of one adapter may stand anywhere.
 *
 *   h_t   = A_l x_t                          (fp32, without the scale; 0 for a token without an adapter)
 *   out_t = base_t + s_l B_l h_t             (base_t for a token without one)
 *
 * and backwards, from the gradient dy_t of out_t:
 *
 *   dh_t = s_l B_l^T dy_t,  dx_t = dx_base_t + A_l^T dh_t,  dA_l = sum_t dh_t x_t^T,  dB_l = s_l sum_t dy_t h_t^T
 *
 * Every sum is taken in fp32.  h and dh enter the matrix units as sums of three BF16 terms, which have their 24 bits (and their sign, so
 * that an infinity among A, B, x or dy comes out as one where it meets a number of 2^-110 at least).
 */
typedef struct {
  int64_t tokens;         /* rows of x, 0 .. 2^24 - 1                                                           */
  int64_t inp, out;       /* columns of x and of the projection's output, multiples of 8 up to 2^22             */
  int64_t adapters, rank; /* 1 .. 2048 adapters of rank 1 .. 128                                                */
  int64_t ld_x;           /* elements from row to row: of x,                                                    */
  int64_t ld_base;        /*   of base (forward) or dx_base (backward),                                         */
  int64_t ld_out;         /*   of out (forward) or dx (backward),                                               */
  int64_t ld_dy;          /*   of dy (backward only); each a multiple of 8, at least the row's length           */
  uint32_t out_dtype;     /* NVFP4_OUT_BF16 or NVFP4_OUT_F32: of base and out (forward only)                    */
} nvfp4_adapters_params;

/* Bytes of workspace that a call with these sizes needs (host arithmetic only; 0 for sizes that the calls refuse).
 *   backward  0: nvfp4_adapters_forward, 1: nvfp4_adapters_backward                                             */
size_t nvfp4_adapters_workspace_bytes(const nvfp4_adapters_params *p, int backward);

/* out = base + adapters.
 *   x          in   [tokens][inp] BF16
 *   base       in   [tokens][out] of out_dtype, or NULL for 0
 *   a, b       in   [adapters][rank][inp] and [adapters][out][rank] BF16, dense
 *   which      in   [tokens] int32
 *   scales     in   [adapters] fp32
 *   h          out  [tokens][rank] fp32, dense, for the backward pass; or NULL
 *   out        out  [tokens][out]; may be base itself (with the same stride, else ERR_SHAPE), no other input
 *   workspace  scratch, 16-byte aligned; holds nothing between calls.  Calls whose work may overlap need one each.
 * Errors: NULL pointer -> ERR_NULL; sizes or strides out of range -> ERR_SHAPE; a buffer that is not 16-byte aligned (which, scales
 * and h: 4 bytes) or a stride that is no multiple of 8 -> ERR_ALIGN; out_dtype, or workspace too small -> ERR_PARAM.  */
int nvfp4_adapters_forward(const void *x, const nvfp4_adapters_params *p, const void *base, const void *a, const void *b,
                           const int32_t *which, const float *scales, float *h, void *out, void *workspace,
                           size_t workspace_bytes, void *stream);

/* The gradients.
 *   dy       in   [tokens][out] BF16
 *   x        in   [tokens][inp] BF16, and h [tokens][rank] as the forward pass left it
 *   dx_base  in   [tokens][inp] BF16: the gradient through the shared projection, or NULL for 0
 *   dx       out  [tokens][inp] BF16; may be dx_base itself (with the same stride, else ERR_SHAPE); NULL if it is not wanted
 *   da, db   out  [adapters][rank][inp] and [adapters][out][rank] fp32, dense; 0 for an adapter without tokens
 * Errors: as above.                                                                                             */
int nvfp4_adapters_backward(const void *dy, const nvfp4_adapters_params *p, const void *x, const float *h, const void *a,
                            const void *b, const int32_t *which, const float *scales, const void *dx_base, void *dx, float *da,
                            float *db, void *workspace, size_t workspace_bytes, void *stream);

/* ---- distillation from a teacher's top logits --------------------------------------------------------------------
 *
 * Per row, with y = logits / temperature and lse = log sum_v exp(y_v): the teacher's list gives p = softmax(teacher / temperature)
 * over its entries (renormalised: the list is all that is known of the teacher), and
 *
 *   loss       = sum_j p_j (log p_j - (y_{i_j} - lse))
 *   dlogits_v  = weight / temperature * (exp(y_v - lse) - sum_{j: i_j = v} p_j)
 *
 * An entry whose index lies outside [0, vocab), or whose teacher logit is -inf, is none.  A row without entries is not learnt from: its
 * loss and its gradient are 0, whatever its logits hold.  Entries with the same index add up.  Logits may be -inf (masked
 * words); at an entry with p_j > 0 that makes the loss infinite, and a row with entries that holds nothing but -inf has no distribution:
 * loss and gradient are NaN, as they are (and lse is) with NaN or +inf among the logits.
 * lse is fp32, and what its rounding leaves (2^-24 |lse|, or all of it where lse is beyond fp32) enters the backward pass'
 * probabilities; loss and step go by differences from the row's largest logit and do without it, so that a row of the type's lowest value
 * alone has its loss and its gradient there.  Neither loss nor gradient is multiplied by temperature^2:
 * `weight` is the place for it.
 */
enum { NVFP4_INDEX_I32 = 0, NVFP4_INDEX_I64 = 1 };

typedef struct {
  int64_t rows;            /* tokens, 0 .. 2^21                                                                */
  int64_t vocab;           /* logits of a row, 1 .. 2^29                                                       */
  int64_t ld;              /* elements from row to row of logits and dlogits, at least vocab, any alignment     */
  int64_t top;             /* entries of a list, 1 .. 1024                                                     */
  float temperature;       /* finite, at least 2^-126 (fp32's least normal number)                          */
  uint32_t x_dtype;        /* NVFP4_X_BF16 or NVFP4_X_F32: of logits and dlogits                               */
  uint32_t teacher_dtype;  /* the same, of teacher                                                             */
  uint32_t index_dtype;    /* NVFP4_INDEX_I32 or NVFP4_INDEX_I64                                               */
} nvfp4_distill_params;

/* loss and lse of every row.
 *   logits   in   [rows][vocab]
 *   teacher  in   [rows][top], dense: the teacher's logits at
 *   index    in   [rows][top], dense
 *   loss     out  [rows] fp32
 *   lse      out  [rows] fp32, or NULL
 * Errors: NULL pointer -> ERR_NULL; sizes out of range -> ERR_SHAPE; a pointer that is not aligned to its elements -> ERR_ALIGN;
 * temperature or a dtype -> ERR_PARAM.                                                                         */
int nvfp4_distill_forward(const void *logits, const nvfp4_distill_params *p, const void *teacher, const void *index,
                          float *loss, float *lse, void *stream);

/* The gradient of sum_t weight_t loss_t.
 *   lse      in   [rows] as nvfp4_distill_forward left it
 *   weight   in   [rows] fp32: the gradient of the rows' losses, or NULL for 1
 *   dlogits  out  [rows][vocab] of x_dtype, stride ld; may be logits itself.  (dlogits - logits) must be a multiple of 16 bytes,
 *                 else ERR_ALIGN
 * Errors: as above.                                                                                             */
int nvfp4_distill_backward(const void *logits, const nvfp4_distill_params *p, const void *teacher, const void *index,
                           const float *lse, const float *weight, void *dlogits, void *stream);

/* Both in one pass: loss (not weighted) and gradient, the logits read once where a row fits the registers of a compute unit. */
int nvfp4_distill_step(const void *logits, const nvfp4_distill_params *p, const void *teacher, const void *index,
                       const float *weight, float *loss, void *dlogits, void *stream);

#ifdef __cplusplus
}
#endif
#endif /* NVFP4_FINETUNE_H */
