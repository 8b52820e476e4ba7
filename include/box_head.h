/*
 * box_head.h -- C ABI of what a detector's heads compute behind the extracted features
 * (libroi_extract.so): dense layers with their epilogue, and the log probabilities of classes.
 *
 * A RoIHead (MMDetection, arXiv 1906.07155, §3.1) takes each RoI's features through shared
 * dense layers to class scores and box deltas, and trains on the log probability of each RoI's
 * class (§3.2).
 *
 * Conventions, status codes, ownership and streams are those of roi_extract.h: every buffer is
 * the caller's, data pointers are device pointers, calls enqueue on `stream` and return without
 * synchronizing, nothing is allocated and no state is kept, argument errors are found on the
 * host before anything is enqueued.  Repeated calls on the same inputs give the same bits.
 *
 * Data of RE_DTYPE_BF16 or RE_DTYPE_F32.  Products of bf16 data are exact and every sum is
 * binary32, and a result is rounded once, when it is stored.
 */
#ifndef BOX_HEAD_H
#define BOX_HEAD_H

#include "roi_extract.h"

#ifdef __cplusplus
extern "C" {
#endif

/* A dense layer, over the rows of x:
 *   t = x weight^T + bias,   y = act(t) + residual
 *   RE_ACT_RELU: max(t, 0) (NaN stays NaN),  RE_ACT_GELU: t Phi(t), Phi the normal distribution's
 *   integral,  RE_ACT_SILU: t / (1 + exp(-t))
 * computed from the binary32 sums t. */
#define RE_ACT_NONE 0
#define RE_ACT_RELU 1
#define RE_ACT_GELU 2
#define RE_ACT_SILU 3
#define RE_LINEAR_MAX_SIZE (1 << 24)      /* inputs and outputs */
typedef struct {
    const void *x;            /* [rows][ins], row stride x_stride (elements) */
    const void *weight;       /* [outs][ins], row stride weight_stride */
    const void *bias;         /* [outs] dense of bias_dtype, or NULL */
    const void *residual;     /* [rows][outs], row stride residual_stride, or NULL */
    int64_t x_stride, weight_stride, residual_stride;
    int64_t rows;             /* may be 0 */
    int64_t ins, outs;        /* at least 1 */
    int32_t dtype;            /* of x, weight, residual, y and the gradients */
    int32_t bias_dtype;       /* RE_DTYPE_F32, or RE_DTYPE_BF16 with bf16 data */
    int32_t act;
} linear_act_t;
/* Any alignment of the element's size.  Fastest where ins, outs and the strides are multiples of 16
 * bytes and the bases are aligned to that.  256 rows of any operand span less than 2^30 bytes, rows, ins
 * and outs are at most 2^31 - 1 and RE_LINEAR_MAX_SIZE, and y, x and weight each have fewer than 2^24
 * blocks of 64 x 64 elements (RE_ERR_UNSUPPORTED). */

/* Device workspace of linear_act_fwd, or of linear_act_bwd where `backward`: partial sums where
 * few results have long sums; in the backward the gradient of t and partial column sums.  Host-only. */
re_status_t linear_act_workspace_size(const linear_act_t *a, int32_t backward, size_t *bytes);

/* y: [rows][outs] dense, no part of it in x, weight or bias; it may be the residual, where that is dense.  slope: the activation's slope at every t, [rows][outs] dense, which the
 * backward takes, or NULL: binary32 with binary32 data; with bf16 data 3 * rows * outs bytes, for
 * numbers c of 24 bits that stand for c * 2^-23 - 1/4 (all ones: NaN), the upper 16 bits of all and then
 * the lower 8 of all, 16-byte aligned.  It has to be NULL for RE_ACT_NONE. */
re_status_t linear_act_fwd(const linear_act_t *a, void *y, void *slope, void *workspace,
                           size_t workspace_bytes, void *stream);

/* Gradients for upstream grad_y ([rows][outs] dense).  With g = grad_y * slope:
 *   grad_x = g weight [rows][ins], grad_weight = g^T x [outs][ins] (both dense),
 *   grad_bias[n] = sum over the rows of g, of bias_dtype, summed before g is rounded to the data's type;
 * the products take g rounded to the data's type (exact for RE_ACT_NONE and RE_ACT_RELU), so that of bf16
 * data grad_x and grad_weight carry one more rounding of each of their terms beside their own;
 * the residual's gradient is grad_y itself.  Each may be NULL (not wanted).  Exactly one of slope
 * (as linear_act_fwd wrote it) and y (RE_ACT_RELU without a residual: what linear_act_fwd wrote) is
 * given, neither with RE_ACT_NONE.  a->residual is not read. */
re_status_t linear_act_bwd(const linear_act_t *a, const void *grad_y, const void *slope, const void *y,
                           void *grad_x, void *grad_weight, void *grad_bias, void *workspace,
                           size_t workspace_bytes, void *stream);

/* Log probabilities over a row's classes.  With x = scale * logits, per row:
 *   lse = log sum_c exp(x_c),  p_c = exp(x_c - lse),
 *   logp = x_label - lse,  entropy = -sum_c p_c log p_c,
 * and the `top` classes of the largest logits, the lower class first among equal ones.  A label
 * outside [0, classes) is not counted: its logp is 0 and has no gradient.  A class whose logit is
 * -inf has p = 0; a row with no other has lse = -inf, logp = -inf, entropy 0 and no gradient.  NaN and
 * +inf make their row's lse, logp and entropy NaN; among the top classes NaN comes first.  A row all of
 * whose logits are at -1e9 has the probabilities that it has with all of them at 0. */
#define RE_LOGPROB_MAX_CLASSES (1 << 24)
#define RE_LOGPROB_MAX_ROWS (1 << 23)     /* divided by a row's parts, of 4088 classes each (RE_ERR_UNSUPPORTED) */
#define RE_LOGPROB_MAX_TOP 16
typedef struct {
    const void *logits;       /* [rows][classes], row stride stride (elements) */
    const int64_t *labels;    /* [rows] dense */
    int64_t stride;
    int64_t rows;             /* may be 0 */
    int64_t classes;          /* at least 1 */
    int32_t dtype;
    int32_t top;              /* in [0, min(classes, RE_LOGPROB_MAX_TOP)] */
    float scale;              /* finite, above 0 */
} class_logprob_t;

/* Device workspace of class_logprob_fwd: the parts of long rows.  Host-only. */
re_status_t class_logprob_workspace_size(const class_logprob_t *a, size_t *bytes);

/* logp, entropy: float[rows]; stats: float[rows][2], the largest x and log sum_c exp(x_c - that), whose
 * sum is lse (-inf and 0 in a row without a class, NaN in one with NaN or +inf), 8-byte aligned; top_logp: float[rows][top],
 * top_index: int64[rows][top], both dense, not used where top is 0. */
re_status_t class_logprob_fwd(const class_logprob_t *a, float *logp, float *entropy, float *stats,
                              float *top_logp, int64_t *top_index, void *workspace,
                              size_t workspace_bytes, void *stream);

/* Gradient of the logits ([rows][classes] dense of dtype) for upstream grad_logp and grad_entropy
 * (float[rows], either may be NULL: zero); stats and entropy as class_logprob_fwd wrote them:
 *   grad_c = scale * (grad_logp ([c = label] - p_c) - grad_entropy p_c (log p_c + entropy)). */
re_status_t class_logprob_bwd(const class_logprob_t *a, const float *grad_logp, const float *grad_entropy,
                              const float *stats, const float *entropy, void *grad_logits, void *stream);

#ifdef __cplusplus
}
#endif

#endif /* BOX_HEAD_H */
