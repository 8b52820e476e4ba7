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
 * bytes and the bases are aligned to that.  256 rows of any operand span less than 2^30 bytes, and
 * rows, ins and outs are at most 2^31 - 1 and RE_LINEAR_MAX_SIZE (RE_ERR_UNSUPPORTED). */

/* Device workspace of linear_act_fwd, or of linear_act_bwd where `backward`: partial sums where
 * few results have long sums; in the backward the gradient of t and partial column sums.  Host-only. */
re_status_t linear_act_workspace_size(const linear_act_t *a, int32_t backward, size_t *bytes);

/* y: [rows][outs] dense.  slope: the activation's slope at every t, [rows][outs] dense, which the
 * backward takes, or NULL: binary32 with binary32 data; with bf16 data 16 bits each, c for
 * c * 2^-15 - 1/4 (65535: NaN).  It has to be NULL for RE_ACT_NONE. */
re_status_t linear_act_fwd(const linear_act_t *a, void *y, void *slope, void *workspace,
                           size_t workspace_bytes, void *stream);

/* Gradients for upstream grad_y ([rows][outs] dense).  With g = grad_y * slope:
 *   grad_x = g weight [rows][ins], grad_weight = g^T x [outs][ins] (both dense),
 *   grad_bias[n] = sum over the rows of g, of bias_dtype, summed before g is rounded to the data's type;
 * the residual's gradient is grad_y itself.  Each may be NULL (not wanted).  Exactly one of slope
 * (as linear_act_fwd wrote it) and y (RE_ACT_RELU without a residual: what linear_act_fwd wrote) is
 * given, neither with RE_ACT_NONE.  a->residual is not read. */
re_status_t linear_act_bwd(const linear_act_t *a, const void *grad_y, const void *slope, const void *y,
                           void *grad_x, void *grad_weight, void *grad_bias, void *workspace,
                           size_t workspace_bytes, void *stream);

#ifdef __cplusplus
}
#endif

#endif /* BOX_HEAD_H */
