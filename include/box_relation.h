/*
 * box_relation.h -- C ABI of the relation head: attention among the boxes of an image,
 * its 8-bit memory of earlier frames, and the norms around it (libroi_extract.so).
 *
 * A detector's RoIHead works on one RoI at a time (MMDetection, arXiv 1906.07155, §3.1);
 * the attention modules among its general components (§2: Generalized Attention, GCNet)
 * relate features to each other.  Here the related things are boxes: the proposals that
 * box_nms_batched selects, [images][max_keep] of them with a count per image on the device,
 * each with features that roi_align_fwd extracted.
 *
 * Conventions, status codes, ownership and streams are those of roi_extract.h: every
 * buffer is the caller's, data pointers are device pointers, calls enqueue on `stream` and
 * return without synchronizing, nothing is allocated and no state is kept, argument errors
 * are found on the host before anything is enqueued, and device-side content (lengths,
 * boxes, masks, page numbers, slots) is never reported as an error but clamped or skipped.
 * Repeated calls on the same inputs give the same bits.
 *
 * Data of RE_DTYPE_BF16 or RE_DTYPE_F32; parameters (bias, weights, gates), their gradients
 * and statistics are binary32.  Products of bf16 data are exact and summed in binary32; the
 * weights of the softmax and the gradient of the logits multiply bf16 data in two parts (all but
 * 2^-17 of them, whatever the size of a call), and every result is rounded once when it is stored.
 */
#ifndef BOX_RELATION_H
#define BOX_RELATION_H

#include "roi_extract.h"

#ifdef __cplusplus
extern "C" {
#endif

#define RE_ATTN_MAX_DIM 128      /* channels of a head: a multiple of 8, at most this */
#define RE_ATTN_MAX_HEADS 256
#define RE_ATTN_MAX_BUCKETS 31   /* per axis */
#define RE_MEMORY_PAGE 32        /* boxes of one page of the memory */

/* Attention of `num_q` query boxes over `num_k` key boxes, per image b and head h; head h
 * reads key head h / (heads / kv_heads):
 *   s_ij = scale * q_i.k_j + bias[h][by(i,j)][bx(i,j)],  p_ij = exp(s_ij - lse_i),
 *   lse_i = log sum_j exp(s_ij),  out_i = sum_j p_ij v_j
 * over the visible keys: j < k_len[b] and k_mask[b][j] != 0.  A row without a visible key
 * (or whose every bias is -inf, see below) has out = 0 and lse = -inf.  Rows i >= q_len[b] are padding:
 * out = 0, lse = -inf, nothing of them is used.  What masked keys and padding hold (NaN and
 * infinities included) has no effect on any result.  An infinity among the values of visible keys
 * makes its channel infinite or NaN.
 *
 * An entry of bias at or below -1e30 (a type's lowest value, say) counts as -inf: its pairs
 * are left out.  Any other is a number: a row whose visible keys are all at -1e9 has the weights
 * that it has with all of them at 0, and the gradients (lse alone is rounded at that size).
 *
 * The bucket of a pair says where the key's centre lies as seen from the query, in units of
 * the query's sides and by octaves: along x, every operation rounded to binary32,
 *   c = (x1 + x2) * 0.5,  inv = 1 / max(x2 - x1, 1),  r = (c_k - c_q) * inv_q,
 *   m = the number of edges <= |r| among the first n = (buckets - 1) / 2 of
 *       2^first_exp * (1 + t/S), t = 0..S-1, S = octave_steps, and so on in every further
 *       octave (n where r is not a number),
 *   bx = n - m where r < 0, else n + m  (by likewise along y).
 */
typedef struct {
    const void *q;            /* [batch][num_q][heads][dim] */
    const void *k, *v;        /* [batch][num_k][kv_heads][dim] */
    int32_t dtype;            /* re_dtype_t of q, k, v (and of out and the gradients) */
    int32_t heads, kv_heads;  /* kv_heads divides heads */
    int32_t dim;
    int64_t batch, num_q, num_k;
    /* element strides of batch, row and head, multiples of 16 bytes (channels are
     * adjacent); bases 16-byte aligned; the rows of one image and 32 more span less than
     * 2^30 bytes (RE_ERR_UNSUPPORTED) */
    int64_t q_stride[3], k_stride[3], v_stride[3];
    float scale;              /* finite, at least 1e-20 */
    int32_t buckets;          /* odd, in [1, RE_ATTN_MAX_BUCKETS]; 0 without bias */
    int32_t first_exp;        /* in [-64, 64] */
    int32_t octave_steps;     /* 1, 2 or 4 */
    const float *bias;        /* [heads][buckets][buckets], or NULL (then the next five
                                 fields are not read) */
    const float *q_boxes;     /* (x1, y1, x2, y2), element strides of batch and row: the
                                 columns 1..4 of RoIs [K][5] serve as they are */
    const float *k_boxes;
    int64_t q_box_stride[2], k_box_stride[2];
    const int32_t *q_len;     /* [batch] valid rows, clamped to [0, num_q]; NULL: all */
    const int32_t *k_len;     /* [batch], clamped to [0, num_k]; NULL: all */
    const uint8_t *k_mask;    /* [batch][num_k], 0: left out; NULL: none */
} box_attn_t;

/* Device workspace of box_attn_fwd and of box_attn_bwd (the larger, where `backward`):
 * partial sums where few rows meet many keys, and in the backward 17 bytes per (row, head)
 * and the bias gradient's partial tables.  May be 0 bytes.  Host-only. */
re_status_t box_attn_workspace_size(const box_attn_t *a, int32_t backward, size_t *bytes);

/* out: [batch][num_q][heads][dim] dense, of a->dtype.  lse: [batch][heads][num_q] or NULL.
 * out_f32: as out in binary32, not rounded, or NULL.  The backward takes sum_c grad_out * out
 * from it where it is given: with a rounded `out` grad_q carries that rounding, which shows where
 * few keys have nearly all of a row's weight.  With out_f32 and no more than RE_ATTN_FEW_KEYS keys
 * the weights multiply bf16 data in three parts, that is whole.
 * workspace: 256-byte aligned. */
#define RE_ATTN_FEW_KEYS 64
re_status_t box_attn_fwd(const box_attn_t *a, void *out, float *lse, float *out_f32,
                         void *workspace, size_t workspace_bytes, void *stream);

/* Gradients for upstream grad_out (dense, as out); out, lse and out_f32 (NULL allowed) as
 * box_attn_fwd wrote them.  With ds_ij = p_ij (grad_out_i.v_j - grad_out_i.out_i):
 *   grad_q_i = scale sum_j ds_ij k_j,  grad_k_j = scale sum_i ds_ij q_i,
 *   grad_v_j = sum_i p_ij grad_out_i (both summed over the heads that share the key head),
 *   grad_bias[h][by][bx] = sum of ds_ij over the pairs of that bucket (all images).
 * All are dense, as q, k, v and bias, and written whole: masked keys and padding get 0.
 * grad_bias: required with a->bias, NULL without. */
re_status_t box_attn_bwd(const box_attn_t *a, const void *grad_out, const void *out,
                         const float *lse, const float *out_f32, void *grad_q, void *grad_k,
                         void *grad_v, float *grad_bias, void *workspace, size_t workspace_bytes,
                         void *stream);

/* Memory of the boxes of earlier frames: keys and values in 8 bits, in pages of
 * RE_MEMORY_PAGE boxes that streams take from one pool in any order.  Slot s is place
 * s % 32 of page s / 32.  For each box and key head, over its channels x (binary32):
 *   a = max |x| over the finite ones,  scale = a / 127,
 *   code = clamp(rint(x / scale), -127, 127), 0 for NaN, and 0 where scale is 0
 * and the value held is code * scale (one binary32 product). */
typedef struct {
    int8_t *k;                /* [num_pages][kv_heads][32][dim] */
    int8_t *v;                /* [num_pages][kv_heads][dim][32] */
    float *k_scale, *v_scale; /* [num_pages][kv_heads][32] */
    float *boxes;             /* [num_pages][32][4] */
    int64_t num_pages;        /* in [1, 2^31) */
    int32_t kv_heads, dim;    /* dim a multiple of 8, at most RE_ATTN_MAX_DIM */
} box_memory_t;               /* all 16-byte aligned */

/* Quantises `count` boxes' k and v ([count][kv_heads][dim], element strides of row and
 * head, channels adjacent, any alignment of the element's size) and writes them with their
 * boxes (float[count][4] dense) to their slots.  slots: int64[count]; a slot outside
 * [0, num_pages * 32) is skipped, and a slot may be named once per call. */
re_status_t box_memory_append(const box_memory_t *m, const int64_t *slots, int64_t count,
                              const void *k, const void *v, int32_t dtype,
                              const int64_t k_stride[2], const int64_t v_stride[2],
                              const float *boxes, void *stream);

/* The values held in `count` slots: k_out, v_out [count][kv_heads][dim] dense of dtype,
 * boxes_out float[count][4]; each may be NULL.  A slot outside the memory reads as 0. */
re_status_t box_memory_read(const box_memory_t *m, const int64_t *slots, int64_t count,
                            void *k_out, void *v_out, int32_t dtype, float *boxes_out,
                            void *stream);

/* Attention of each stream's query boxes over what the stream remembers: as box_attn_fwd
 * with the keys, values and boxes held in places 0 .. lengths[b] - 1 of the stream's
 * pages[b][0 .. max_pages - 1] (place t: page t / 32).  Places of a page number outside
 * [0, num_pages) are left out. */
typedef struct {
    const void *q;            /* [batch][num_q][heads][dim] */
    int32_t dtype;
    int32_t heads;            /* a multiple of the memory's kv_heads */
    int64_t batch, num_q, max_pages;
    int64_t q_stride[3];      /* as box_attn_t */
    float scale;
    int32_t buckets, first_exp, octave_steps;
    const float *bias;        /* as box_attn_t */
    const float *q_boxes;
    int64_t q_box_stride[2];
    const int32_t *q_len;     /* [batch] or NULL */
    const int32_t *pages;     /* [batch][max_pages] */
    const int32_t *lengths;   /* [batch], clamped to [0, 32 * max_pages] */
} box_recall_t;

re_status_t box_memory_attn_workspace_size(const box_memory_t *m, const box_recall_t *r,
                                           size_t *bytes);
/* out: [batch][num_q][heads][dim] dense of r->dtype; lse: [batch][heads][num_q] or NULL. */
re_status_t box_memory_attn_fwd(const box_memory_t *m, const box_recall_t *r, void *out,
                                float *lse, void *workspace, size_t workspace_bytes,
                                void *stream);

/* The norms around a block, its gate and the residual sum, in one pass:
 *   y = x + alpha * gate * N1(branch),   u = N2(y)
 *   RE_NORM_RMS:    N(t) = t / sqrt(mean(t^2) + eps) * weight
 *   RE_NORM_LAYER:  N(t) = (t - mean(t)) / sqrt(var(t) + eps) * weight + bias
 * over the channels of a row, in binary32; u is made from y before y is rounded.
 * Gate row g serves rows g * (rows / gates) and following. */
#define RE_NORM_RMS 0
#define RE_NORM_LAYER 1
#define RE_NORM_MAX_CHANNELS 8192
typedef struct {
    const void *x;            /* [rows][channels], row stride x_stride (elements) */
    const void *branch;       /* as x, or NULL: y = x, only the second norm */
    int64_t x_stride, branch_stride;
    int32_t dtype, norm;
    int64_t rows;
    int32_t channels;         /* in [1, RE_NORM_MAX_CHANNELS] */
    float alpha, eps;         /* finite, eps > 0 */
    int64_t gates;            /* divides rows; 0 without a gate */
    const float *gate;        /* [gates][channels] or NULL (1) */
    const float *post_weight, *post_bias;   /* N1: [channels], NULL: 1 and 0 */
    const float *pre_weight, *pre_bias;     /* N2: [channels], NULL: 1 and 0 */
} gated_norm_t;

/* y, u: [rows][channels] dense of dtype; y may be NULL without a branch (it is x then), u
 * may be NULL (no second norm).  stats: float[rows][4] (mean and 1/sqrt of N1, of N2), or
 * NULL; entries of a norm that is left out are 0. */
re_status_t gated_norm_fwd(const gated_norm_t *a, void *y, void *u, float *stats, void *stream);

/* Device workspace of gated_norm_bwd: partial column sums. */
re_status_t gated_norm_workspace_size(const gated_norm_t *a, size_t *bytes);

/* Gradients for upstream grad_y and grad_u ([rows][channels] dense of dtype; either may be
 * NULL: zero).  stats as gated_norm_fwd wrote them.  grad_x, grad_branch: dense of dtype;
 * grad_gate [gates][channels]; the others [channels].  Each may be NULL (not wanted). */
typedef struct {
    void *x, *branch;
    float *gate, *post_weight, *post_bias, *pre_weight, *pre_bias;
} gated_norm_grads_t;
re_status_t gated_norm_bwd(const gated_norm_t *a, const void *grad_y, const void *grad_u,
                           const float *stats, const gated_norm_grads_t *grads, void *workspace,
                           size_t workspace_bytes, void *stream);

#ifdef __cplusplus
}
#endif

#endif /* BOX_RELATION_H */
