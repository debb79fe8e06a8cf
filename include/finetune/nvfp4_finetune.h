/*
 * nvfp4_finetune -- recovering, and serving, a model whose weights are quantized to NVFP4 (same library and
 * conventions as nvfp4_46.h: device pointers, caller's memory and stream, an nvfp4_status back, nothing enqueued
 * by a call that is refused).
 *
 *   nvfp4_adapters_*   low-rank adapters of many requests at once, beside a projection that they share: the weight stays
 *                      quantized and frozen, adapters hold the correction
 *   nvfp4_distill_*    the divergence of a model's logits from a teacher's top logits, and its gradient
 *   nvfp4_weight_product, nvfp4_experts_*   activations as they are times a quantized weight, or those of many experts; tokens to
 *                      their experts and back
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

/* ---- products with a quantized weight and activations as they are -----------------------------------------------------
 *
 * W is NVFP4, as nvfp4_46_quantize leaves it: W[n][k] = alpha * value(code[n][k]) * value(scale[n][k / 16]).  x is BF16 or fp32 and enters
 * unrounded (nvfp4_46_gemm takes it quantized too):
 *
 *   out[s][n] = alpha sum_k x[row(s)][k] value(code[n][k]) value(scale[n][k / 16])
 *
 * A weight's value without alpha has six significant bits at most and is exact in BF16, fp32 activations are sums of three BF16 terms (all 24
 * bits from 2^-110 up; below, what is less than 2^-133 is lost), so products are exact; sums are fp32's, in a fixed order that depends on sizes
 * alone.  For the gradient dx = dy W pass the packing
 * of the transposed weight (columnwise codes and scales; with block2d they hold the same values).
 *
 * nvfp4_experts_product does so with a weight for each expert: the rows begin[e] .. begin[e + 1] - 1 of out are expert e's.  A row in front
 * of the first expert's or behind the last one's, and one whose token is none of x's rows, is 0.
 */
typedef struct {
  int64_t rows;           /* rows of x, 0 .. 2^24 - 1                                                           */
  int64_t inp, out;       /* K, a multiple of 32 up to 2^22, and N, 1 .. 2^22                                   */
  int64_t experts;        /* 1 .. 1024 (nvfp4_weight_product: 1)                                                */
  int64_t slots;          /* rows of out, 0 .. 2^30 (nvfp4_weight_product, or without `token`: as many as x's)  */
  int64_t ld_x, ld_out;   /* elements from row to row of x (a multiple of 8, at least K) and of out (at least N) */
  uint32_t x_dtype;       /* NVFP4_X_BF16 or NVFP4_X_F32                                                        */
  uint32_t out_dtype;     /* NVFP4_OUT_BF16 or NVFP4_OUT_F32                                                    */
  uint32_t flags;         /* 0 or NVFP4_GEMM_B_TILE_SCALES: scales [N/16][K/16] (N a multiple of 16)            */
} nvfp4_product_params;

/*   x       in   [rows][K]
 *   codes   in   [N][K/2], dense
 *   scales  in   [N][K/16], dense, each byte <= 0x7E
 *   alpha   in   1 float (device)
 *   out     out  [rows][N]; may not overlap an input
 * Errors: NULL pointer -> ERR_NULL; sizes or strides out of range -> ERR_SHAPE; a buffer that is not 16-byte aligned (alpha: 4) or ld_x no
 * multiple of 8 -> ERR_ALIGN; a dtype or flags -> ERR_PARAM.                                                    */
int nvfp4_weight_product(const void *x, const nvfp4_product_params *p, const void *codes, const void *scales, const float *alpha,
                         void *out, void *stream);

/*   token   in   [slots] int32: the row of x that a row of out is made of, or NULL: row s of x
 *   begin   in   [experts + 1] int32, not falling, within 0 .. slots (device)
 *   codes, scales, alpha  in  [experts] of each, one after the other
 * Errors: as above (token, begin: 4 bytes).                                                                     */
int nvfp4_experts_product(const void *x, const nvfp4_product_params *p, const int32_t *token, const int32_t *begin,
                          const void *codes, const void *scales, const float *alpha, void *out, void *stream);

/* ---- tokens to their experts, and back --------------------------------------------------------------------------------
 *
 * Token t has the experts ids[t][j], j < top; an id outside [0, experts) is none.  An expert may stand twice.  The pairs (t, j) are put in
 * the order of their experts, within an expert by t and then j; those without an expert come last.  There are tokens * top places ("slots").
 *
 *   place[t][j]   the pair's slot i, or -1 - i for a pair without an expert
 *   token[i]      the token of slot i, or -1 where the pair has no expert
 *   begin[e]      the first slot of expert e; begin[experts] the first behind the last expert's
 *
 *   spread    xs[i] = x_t at every slot i = place[t][j], 0 at the slots of pairs without an expert
 *   combine   y_t = base_t + sum_j weights[t][j] ys[place[t][j]] over the pairs that have an expert; without weights they are 1, and
 *             this is spread's gradient
 *   backward  dys[place[t][j]] = weights[t][j] dy_t (0 at the slots of pairs without an expert),
 *             dweights[t][j] = sum_c dy_t[c] ys[place[t][j]][c] (0 for such a pair); base's gradient is dy
 *
 * Sums are fp32's, over j and over the columns in a fixed order.  A place that is no slot is left out.
 */
typedef struct {
  int64_t tokens, top;    /* 0 .. 2^24 - 1 tokens of 1 .. 64 experts each                                       */
  int64_t experts;        /* 1 .. 1024 (sort only)                                                              */
  int64_t width;          /* columns, a multiple of 8 up to 2^22 (all but sort)                                 */
  int64_t ld_token;       /* elements from row to row: of x, y, dy,                                             */
  int64_t ld_base;        /*   of base,                                                                         */
  int64_t ld_slot;        /*   of xs, ys,                                                                       */
  int64_t ld_dslot;       /*   of dys; each a multiple of 8, at least width                                     */
  uint32_t token_dtype;   /* NVFP4_X_BF16 or NVFP4_X_F32: of x, y, base, dy                                     */
  uint32_t slot_dtype;    /* the same, of xs, ys, dys                                                           */
  uint32_t index_dtype;   /* NVFP4_INDEX_I32 or NVFP4_INDEX_I64: of ids (sort only)                             */
} nvfp4_experts_params;

/* Bytes of workspace that nvfp4_experts_sort needs (host arithmetic only; 0 for sizes that it refuses; at least 16).           */
size_t nvfp4_experts_workspace_bytes(const nvfp4_experts_params *p);

/*   ids        in   [tokens][top], dense
 *   place      out  [tokens][top] int32, dense
 *   token      out  [tokens * top] int32
 *   begin      out  [experts + 1] int32
 *   workspace  scratch, 16-byte aligned; holds nothing between calls.  Calls whose work may overlap need one each.  Where 16 bytes are
 *              enough, they are left alone.
 * No output may overlap ids or another output.
 * Errors: NULL pointer -> ERR_NULL; sizes out of range -> ERR_SHAPE; a pointer that is not aligned to its elements -> ERR_ALIGN;
 * index_dtype, or workspace too small -> ERR_PARAM.                                                             */
int nvfp4_experts_sort(const void *ids, const nvfp4_experts_params *p, int32_t *place, int32_t *token, int32_t *begin,
                       void *workspace, size_t workspace_bytes, void *stream);

/*   x   in   [tokens][width]            xs  out  [tokens * top][width]
 * Errors: NULL pointer -> ERR_NULL; sizes or strides out of range -> ERR_SHAPE; a buffer that is not 16-byte aligned (place,
 * weights: 4) or a stride that is no multiple of 8 -> ERR_ALIGN; a dtype -> ERR_PARAM.                          */
int nvfp4_experts_spread(const void *x, const nvfp4_experts_params *p, const int32_t *place, void *xs, void *stream);

/*   ys       in   [tokens * top][width]
 *   weights  in   [tokens][top] fp32, dense, or NULL for 1
 *   base     in   [tokens][width], or NULL for 0
 *   y        out  [tokens][width]; may be base itself (with the same stride, else ERR_SHAPE), no other input
 * Errors: as above.                                                                                             */
int nvfp4_experts_combine(const void *ys, const nvfp4_experts_params *p, const int32_t *place, const float *weights,
                          const void *base, void *y, void *stream);

/*   dy        in   [tokens][width]
 *   dys       out  [tokens * top][width]; may be ys itself (with the same stride, else ERR_SHAPE), no other input
 *   dweights  out  [tokens][top] fp32, dense
 * Errors: as above.                                                                                             */
int nvfp4_experts_combine_backward(const void *dy, const nvfp4_experts_params *p, const void *ys, const int32_t *place,
                                   const float *weights, void *dys, float *dweights, void *stream);

#ifdef __cplusplus
}
#endif
#endif /* NVFP4_FINETUNE_H */
