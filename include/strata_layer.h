/*
 * strata_layer.h -- the operators of an MoE layer around the routing path of strata_moe.h: the router that makes
 * the expert ids and gate weights, the residual addition with root-mean-square norm that makes x (in bf16 or in
 * 8 bits), the row quantiser, and the experts' products over the receive buffer in 8 bits.
 *
 * The conventions of strata_moe.h hold: every function returns a strata_status, checks what the host can see
 * before it launches anything, enqueues its kernels on the given stream without synchronising, and allocates no
 * device memory.  Errors that only the device can see go to the context's status word.  Tensors are row-major;
 * a "stride" is the distance between two rows, in elements of that tensor, and may exceed the row's length.
 * Rounding to bf16 and to 8-bit codes is to nearest, ties to even.  All sums, norms, softmax statistics and
 * scales are binary32 (the products of int8 rows accumulate in int32, exactly).
 * Functions and quotients inside are binary32 as well.  Where they are coarser than expf and a rounded quotient (by CUDA's
 * bounds, in units of the last place of binary32): the gradient of softmax weights that are not renormalised, for bf16
 * logits: an exponential within 2 + 1.2 |l - max|; silu in a gated product: an exponential within 2 + 1.2 |g| and a division within
 * 2, and zero where g is below -87.3; the norm's gradient: a reciprocal square root within 2; the balance loss and
 * its gradient: a sigmoid's reciprocal within 1; the gradient alone, for bf16 logits: an exponential as in the router's.  The router decides a token
 * in one of two ways, whose weights may differ in the last places.
 * The order of a row's sums depends on the rows and columns of the call: equal calls give equal bits, but the last bit of a row's norm
 * may differ between a call that holds it among few rows and one that holds it among many.
 * strata_ctx_set_sm_budget bounds the grids of the experts' products, which choose their tile by it as well; in int8 and in 4 bits that
 * does not show in the results.  The other operators size their grids for the whole GPU.
 */
#ifndef STRATA_LAYER_H
#define STRATA_LAYER_H

#include "strata_moe.h"

#ifdef __cplusplus
extern "C" {
#endif

/* Element types of the operands below. */
typedef enum {
    STRATA_T_BF16 = 0,
    STRATA_T_F32 = 1,
    STRATA_T_INT8 = 2,             /* codes -127..127, largest magnitude of a row = 127       */
    STRATA_T_E4M3 = 3,             /* e4m3 ("fn"), largest magnitude of a row = 448           */
    STRATA_T_MXF4 = 4,             /* rows in 4 bits, see strata_rows4                        */
    STRATA_T_NVF4 = 5
} strata_type;

/* ---- router ----------------------------------------------------------------------------------------------
 * scores   s = softmax(logits) over the row's experts, or 1 / (1 + exp(-logits)) elementwise
 * choice   c = s + bias (binary32); without a bias, and unless groups score by a sum, the logits themselves are
 *          compared, which is the same order without the ties that rounding makes.  The bias takes part in the
 *          choice only (load balancing), never in the weights.
 * groups   n_group > 1: the E experts form n_group equal runs; a group scores the largest c of its experts
 *          (STRATA_GROUP_MAX) or the sum of its two largest (STRATA_GROUP_TOP2); the topk_group best groups
 *          stay, ties to the lower group
 * ids      the K experts of largest c, in decreasing order, ties to the lower index
 * weights  w_k = scale * s[id_k], divided by the sum of the token's K scores if renormalise is set (for the softmax: scale times
 *          the softmax over the chosen logits, so that chosen scores below the range of binary32 count as well)
 * An expert whose logit (or whose choice) is NaN or -inf is never chosen, and a NaN or -inf logit counts as a
 * score of zero in the softmax.  A token with fewer than K such experts left gets id -1 and weight 0 in its last
 * slots (the layout treats -1 as "not routed" under STRATA_FLAG_ALLOW_UNROUTED).  If every chosen sigmoid score is
 * zero, renormalised weights are zero. */
#define STRATA_SCORE_SOFTMAX 0
#define STRATA_SCORE_SIGMOID 1
#define STRATA_GROUP_MAX 0
#define STRATA_GROUP_TOP2 1
typedef struct {
    int32_t score;                 /* STRATA_SCORE_*                                          */
    int32_t renormalise;           /* 0 or 1                                                  */
    int32_t n_group;               /* 1 = no groups; divides E; at most 32                    */
    int32_t topk_group;            /* 1..n_group, topk_group * E / n_group >= K               */
    int32_t group_score;           /* STRATA_GROUP_*                                          */
    float scale;                   /* finite                                                  */
} strata_route_params;

/* logits: device, bf16 or float [R*T, E] with row stride logits_stride >= E; bias: device float [E] or NULL;
 * topk_ids: device int32 [R,T,K]; topk_w: device float [R,T,K], as the layout and combine take them.  R, T, E, K
 * are the context's.  One launch. */
strata_status strata_moe_route(strata_ctx *ctx, const strata_route_params *params, const void *logits,
                               int32_t logits_type, int64_t logits_stride, const float *bias, int32_t *topk_ids,
                               float *topk_w, void *stream);

/* Gradient of the logits from the gradient of the weights (the choice itself has none):
 *   d_k = scale * dw_k, or with renormalised weights (scale / D) * (dw_k - sum_j dw_j s_j / D), D = sum_j s_j
 *   sigmoid: dlogit = d * s * (1 - s);  softmax: dlogit_e = s_e * (d_e - sum_k d_k s_k), d_e = 0 if not chosen
 * topk_ids are the forward call's; -1 is skipped, a repeated id adds up, an id outside [0,E) is skipped and
 * raises BAD_EXPERT_ID.  If D is zero (sigmoid) the gradient is zero; a NaN or -inf logit gets zero.  dlogits has the
 * type of logits and row stride dlogits_stride; every element of its rows is written.  Needs a workspace (the
 * status word).  One launch. */
strata_status strata_moe_route_grad(strata_ctx *ctx, const strata_route_params *params, const void *logits,
                                    int32_t logits_type, int64_t logits_stride, const int32_t *topk_ids,
                                    const float *dtopk_w, void *dlogits, int64_t dlogits_stride, void *stream);

/* ---- residual addition and root-mean-square norm ------------------------------------------------------------
 * h = bf16(x + residual) if residual is given (written to residual_out, which may be residual itself), else x
 * y = (h * weight) * rstd,  rstd = 1 / sqrt(mean(h^2) + eps): the mean is of h as it is stored
 * out  (bf16) = bf16(y), if given
 * q (8 bits)  = codes of y * limit / max|y|, q_scale[row] = max|y| / limit, limit = 127 (int8) or 448 (e4m3), if
 *               given: y is about code * q_scale.  With bf16 weights the quotient is one correctly rounded binary32 value
 *               before it becomes a code, so half-way cases go to the even code; with float weights h * weight and its multiple
 *               by limit are rounded first, 2^-23 relative in all.  Codes of an all-zero row are zero with scale 0, whatever eps.
 *               Codes are of y, not of bf16(y); they do not depend on rstd, which cancels.
 * NaN and infinities follow the formula in `out` (eps = 0 makes rstd infinite where the squares sum to zero or underflow to it);
 * codes and scale of a row that holds one are unspecified.
 * x, residual, residual_out, out: device bf16, 16-byte aligned, strides multiples of 8; weight: device bf16 or float
 * [cols], 16-byte aligned; q: 8-byte aligned, stride a multiple of 8; q_scale: element `row` at q_scale[row *
 * q_scale_stride].  cols: a multiple of 8, at most 32768.  rows may be 0 (nothing is launched, row
 * tensors may be NULL).  One of out and q is
 * required.  residual and residual_out come together.  eps >= 0.  Outputs may alias no input, except residual_out
 * = residual or x, and out = x.  One launch. */
typedef struct {
    int64_t rows;
    int32_t cols;
    int32_t weight_type;           /* STRATA_T_BF16 or STRATA_T_F32                           */
    float eps;
    int32_t q_type;                /* STRATA_T_INT8 or STRATA_T_E4M3 (read if q is given)     */
    const void *x;
    const void *residual;          /* NULL: no addition                                       */
    const void *weight;
    void *residual_out;
    void *out;
    void *q;
    float *q_scale;
    int64_t x_stride, residual_stride, residual_out_stride, out_stride, q_stride, q_scale_stride;
} strata_norm_args;
strata_status strata_norm(strata_ctx *ctx, const strata_norm_args *args, void *stream);

/* Backward pass of out: g = dy * weight, hat = h * rstd,
 *   dx = rstd * (g - hat * mean(g * hat)) + dresidual      (dx is the gradient of x and of residual alike)
 *   dweight[c] = sum over rows of dy * hat                 (float; the order of the sum is fixed)
 * h: the stored sum (residual_out of the forward pass, or x where there was no residual); dresidual: the gradient
 * that arrives at residual_out, or NULL.  dx may be dy or dresidual.  scratch: device, 16-byte aligned, of
 * strata_norm_grad_scratch_bytes.  rows = 0: dweight is zeroed.  Needs a workspace (the status word).  Two launches. */
typedef struct {
    int64_t rows;
    int32_t cols;
    int32_t weight_type;
    float eps;
    int32_t reserved;
    const void *dy;
    const void *h;
    const void *weight;
    const void *dresidual;
    void *dx;
    float *dweight;
    void *scratch;
    size_t scratch_bytes;
    int64_t dy_stride, h_stride, dresidual_stride, dx_stride;
} strata_norm_grad_args;
strata_status strata_norm_grad_scratch_bytes(strata_ctx *ctx, int64_t rows, int32_t cols, size_t *bytes);
strata_status strata_norm_grad(strata_ctx *ctx, const strata_norm_grad_args *args, void *stream);

/* ---- rows to 8 bits -----------------------------------------------------------------------------------------
 * q = codes of x * limit / max|x|, q_scale[row] = max|x| / limit, as in strata_norm with a weight of 1.  n_valid: device int32, or NULL;
 * if given, only rows below *n_valid are read and written (expert_offset + E of a layout: the rows in use of a
 * receive buffer).  Alignments, strides and limits as in strata_norm.  One launch. */
strata_status strata_quantize_rows(strata_ctx *ctx, const void *x, int64_t x_stride, int64_t rows, int32_t cols,
                                   int32_t q_type, void *q, int64_t q_stride, float *q_scale, int64_t q_scale_stride,
                                   const int32_t *n_valid, void *stream);

/* ---- the experts' products ------------------------------------------------------------------------------------
 * For every expert e and every row r of its segment (expert_offset[e] .. + expert_count[e] of the layout; all
 * R*slot_capacity rows of the segment in the fixed-capacity layout, empty slots too):
 *   y[r, n] = (sum_k a[r,k] * w[e,n,k]) * (a_scale[r] * w_scale[e,n])
 *   out[r, n] = bf16(y[r, n])                                             n < channels, or
 *   out[r, n] = bf16(silu(y[r, n]) * y[r, channels/2 + n])                n < channels/2, if gated
 * a: 8-bit rows [a_rows, inner], 16-byte aligned, stride in bytes a multiple of 16, a_rows >= strata_moe_recv_rows;
 * a_scale of row r at a_scale[r * a_scale_stride]; w: [E, channels, inner] contiguous, 16-byte aligned; w_scale: float
 * [E, channels]; out: bf16 (stored in pairs where out, out_stride and the channels of out are even multiples of two bytes,
 * one by one otherwise).  inner: a multiple of 16, at most 131056 (int32 sums cannot overflow); channels: any number, an even
 * one if gated.  Rows outside the segments (padding, unrouted) are not written.
 * Needs a workspace (the status word).  One launch. */
typedef struct {
    int32_t type;                  /* STRATA_T_INT8 or STRATA_T_E4M3, of a and w alike        */
    int32_t gated;                 /* 0 or 1: w holds the gate's channels/2 rows, then up's   */
    int32_t inner;
    int32_t channels;
    int64_t a_rows;
    const void *a;
    const float *a_scale;
    const void *w;
    const float *w_scale;
    void *out;
    int64_t a_stride, a_scale_stride, out_stride;
} strata_matmul_args;
strata_status strata_moe_expert_matmul(strata_ctx *ctx, const strata_moe_layout_t *layout,
                                       const strata_matmul_args *args, void *stream);

/* ---- rows in 4 bits ------------------------------------------------------------------------------------------
 * A value is an e2m1 code (0, 0.5, 1, 1.5, 2, 3, 4, 6 and their negatives), times the scale of its block, times the scale of its
 * row if there is one.  Two codes share a byte, the first in its low half.
 *   MXF4: blocks of 32 values, a scale byte s stands for 2^(s - 127), 255 for NaN (e8m0)
 *   NVF4: blocks of 16 values, the scale is an e4m3 number, not negative
 * codes: row r at byte r * code_stride, cols / 2 bytes; block: scale bytes, row r at byte r * block_stride, cols / 32 or
 * cols / 16 bytes; scale: float, row r at scale[r * scale_stride], or NULL (1).  codes and block are 16-byte aligned, their strides
 * multiples of 16 that hold a row, below 2^40.  cols is a multiple of 32. */
typedef struct {
    void *codes;
    void *block;
    float *scale;
    int64_t code_stride, block_stride, scale_stride;
} strata_rows4;

/* Codes and scales of bf16 rows (M: a block's largest magnitude, A: the row's):
 *   MXF4: the power of two 2^s, s = floor(log2 M) - 2, and one more where M >= 7 * 2^s; between 2^-127 and 2^125;
 *         codes of x / 2^s.  scale must be NULL.
 *   NVF4: scale[row] = A / 2688 (one binary32 division); block scale b = e4m3(448 M / A); codes of 2688 x / (A b), zero where
 *         b is zero.  scale is required.
 * Every code and block scale is the nearest to the exact quotient, ties to even, 6 (and 448) at the most.  A block of zeros has zero
 * codes, with block scale 0.  A block (MXF4) or row (NVF4) that holds a NaN or an infinity stands for NaN throughout; its
 * codes are unspecified.  Below A = 2688 * 2^-126 the row's scale is a subnormal number and loses places.
 * n_valid: as in strata_quantize_rows.  x: bf16, 16-byte aligned, stride a multiple of 8.  cols <= 32768.  rows may
 * be 0.  Outputs may alias no input.  One launch. */
strata_status strata_quantize_rows4(strata_ctx *ctx, const void *x, int64_t x_stride, int64_t rows, int32_t cols,
                                    int32_t type, const strata_rows4 *q, const int32_t *n_valid, void *stream);

/* out = the values of 4-bit rows, code * (block scale * scale) with each product rounded to binary32, in bf16 or float (out_type).
 * out: 16-byte aligned, stride a multiple of 16 bytes.  One launch. */
strata_status strata_dequantize_rows4(strata_ctx *ctx, const strata_rows4 *q, int64_t rows, int32_t cols, int32_t type,
                                      void *out, int32_t out_type, int64_t out_stride, const int32_t *n_valid, void *stream);

/* The experts' products over 4-bit rows: as strata_moe_expert_matmul, with
 *   y[r, n] = (sum_k a[r,k] * w[e,n,k]) * (scale[r] * w.scale[e,n])
 * where a and w include their block scales.  a: the rows of the receive buffer; w: [E, channels] rows in order (row e * channels
 * + n), of the same type, with a scale per channel (a scale per expert is spread over its channels) or none.  inner: a multiple of
 * 32, at most 131072; channels: any number, an even one if gated.  The sums are binary32.  Needs a workspace (the status word).
 * One launch. */
typedef struct {
    int32_t type;                  /* STRATA_T_MXF4 or STRATA_T_NVF4, of a and w alike        */
    int32_t gated;                 /* 0 or 1: w holds the gate's channels/2 rows, then up's   */
    int32_t inner;
    int32_t channels;
    int64_t a_rows;
    strata_rows4 a, w;
    void *out;                     /* bf16, as in strata_moe_expert_matmul                    */
    int64_t out_stride;
} strata_matmul4_args;
strata_status strata_moe_expert_matmul4(strata_ctx *ctx, const strata_moe_layout_t *layout,
                                        const strata_matmul4_args *args, void *stream);

/* ---- balance of the router -------------------------------------------------------------------------------------
 * The R*T tokens form one group, or one per source rank (per_rank).  A token takes part if one of its K ids is routed (not
 * -1); the others are padding.  For a group of n such tokens, C[e] slots of them routed to expert e:
 *   p[t, e] = softmax(logits[t])[e], or the sigmoid scores of the token over their sum
 *   prob[e] = (sum_t p[t, e]) / n          (0 where n is 0)
 *   balance = weight * mean over the groups with tokens of  sum_e (E * C[e] / (K * n)) * prob[e]
 *   z       = z_weight * mean over all tokens that take part of  log(sum_e exp(logits[t, e]))^2
 * A NaN or -inf logit counts as a score of zero, as in the router; a token without any other logit adds nothing to prob and z.
 * C is a constant of the gradient.  loss[0] = balance, loss[1] = z; both are 0 where no token takes part.
 * An id outside [0,E) other than -1 is not counted and raises BAD_EXPERT_ID.  The order of all sums is fixed by the shape. */
typedef struct {
    int32_t score;                 /* STRATA_SCORE_*                                          */
    int32_t per_rank;              /* 0: one group, 1: R groups                               */
    float weight;                  /* finite                                                  */
    float z_weight;                /* finite                                                  */
} strata_balance_params;
typedef struct {                   /* device, what the gradient needs of the forward call     */
    int32_t *count;                /* [groups, E]  C                                          */
    int32_t *tokens;               /* [groups]     n                                          */
    float *prob;                   /* [groups, E]                                             */
} strata_balance_stats;

/* logits, topk_ids as in strata_moe_route (logits may be any row-strided bf16 or float rows [R*T, E]); loss: device float
 * [2]; scratch: device, 16-byte aligned, of strata_moe_balance_scratch_bytes.  Needs a workspace.  One launch where an expert
 * has few partial sums (groups of up to 2,048 tokens at 32 experts or fewer, of 256 above 128), else two. */
strata_status strata_moe_balance_scratch_bytes(strata_ctx *ctx, const strata_balance_params *params, size_t *bytes);
strata_status strata_moe_balance_loss(strata_ctx *ctx, const strata_balance_params *params, const void *logits,
                                      int32_t logits_type, int64_t logits_stride, const int32_t *topk_ids, float *loss,
                                      const strata_balance_stats *stats, void *scratch, size_t scratch_bytes, void *stream);

/* dlogits = dloss[0] * d balance / d logits + dloss[1] * d z / d logits + add, of the type of logits.  dloss: device float
 * [2], or NULL (1, 1); add: a gradient that arrives otherwise (strata_moe_route_grad), of the type of logits, or NULL; dlogits may be
 * add.  stats: as strata_moe_balance_loss wrote them for the same ids.  Padding tokens and masked logits get `add`, or 0.  Every
 * element of dlogits' rows is written.  One launch. */
strata_status strata_moe_balance_grad(strata_ctx *ctx, const strata_balance_params *params, const void *logits,
                                      int32_t logits_type, int64_t logits_stride, const int32_t *topk_ids,
                                      const strata_balance_stats *stats, const float *dloss, const void *add,
                                      int64_t add_stride, void *dlogits, int64_t dlogits_stride, void *stream);

#ifdef __cplusplus
}
#endif
#endif /* STRATA_LAYER_H */
