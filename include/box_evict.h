/*
 * box_evict.h -- C ABI of what a memory of boxes forgets (libroi_extract.so): the attention that
 * each remembered box has received, and the boxes of least weight making room.
 *
 * The memory is that of box_relation.h, whose conventions hold here too.
 */
#ifndef BOX_EVICT_H
#define BOX_EVICT_H

#include "box_relation.h"

#ifdef __cplusplus
extern "C" {
#endif

/* The attention that the remembered boxes receive from a frame's queries, added up:
 *   weight_out[b][t] = decay * weight[b][t] + sum over heads h and rows i < q_len[b] of
 *                      min(exp(s_it - lse[b][h][i]), 1)
 * for the places t < lengths[b] of a page inside the memory, s as box_memory_attn_fwd computes it;
 * 0 for every other place.  weight, weight_out: float[batch][32 * max_pages], which may be the same
 * buffer; weight may be NULL (zeros; decay is then not used).  lse: float[batch][heads][num_q], as
 * box_memory_attn_fwd wrote it, or the log sum of a softmax over more keys than these; a row whose
 * lse is not finite adds nothing, whatever its query and biases hold, and a logit that is NaN in a row whose
 * lse is finite adds nothing.  exp(s - lse) is as exact as lse is: its relative error is up to
 * 2^-23 |lse| more than that of the difference.  decay: finite. */
re_status_t box_memory_weigh(const box_memory_t *m, const box_recall_t *r, const float *lse,
                             const float *weight, float decay, float *weight_out, void *stream);

/* Each stream keeps the min(keep[b], lengths[b]) boxes of the largest weight, of equal ones those in
 * lower places, NaN counting as larger than any number.  They end in its first places: those that were
 * there stay where they are, and those further on go, in the order of their places, to the places that
 * became free, in order; every other place holds what it held (pages that boxes come to are written
 * whole, and nothing else may write to them meanwhile).
 *   lengths_out[b]: the boxes kept;  weight_out[b][t]: the weight of the box that is now in place t,
 *   0 from lengths_out[b] on;  origin[b][t]: the place that it was in, -1 from there on.
 * A stream that has a page number outside [0, num_pages) among the pages of its lengths[b] places
 * is left as it is (origin[b][t] = t).  lengths is clamped to [0, 32 * max_pages], keep to
 * [0, lengths[b]].  A page belongs to one stream and is named once in its row.  Fewer than 2^24 pages
 * times (kv_heads + 3) / 4, and at most 2^21 streams (RE_ERR_UNSUPPORTED); box_memory_weigh takes fewer than 2^22
 * pages. */
typedef struct {
    int64_t batch, max_pages;
    const int32_t *pages;     /* [batch][max_pages] */
    const int32_t *lengths;   /* [batch] */
    const int32_t *keep;      /* [batch] */
    const float *weight;      /* [batch][32 * max_pages] */
} box_evict_t;

/* Device workspace of box_memory_evict: places that become free, and where boxes go.  Host-only. */
re_status_t box_memory_evict_workspace_size(const box_memory_t *m, const box_evict_t *e, size_t *bytes);
/* lengths_out: int32[batch], may be e->lengths; weight_out: float[batch][32 * max_pages], not
 * e->weight; origin: int32[batch][32 * max_pages], or NULL. */
re_status_t box_memory_evict(const box_memory_t *m, const box_evict_t *e, int32_t *lengths_out,
                             float *weight_out, int32_t *origin, void *workspace,
                             size_t workspace_bytes, void *stream);

#ifdef __cplusplus
}
#endif

#endif /* BOX_EVICT_H */
