// relation_api.hip -- the C ABI declared in include/box_relation.h.
//
// As in api.hip, every argument is checked on the host before anything is enqueued, and no
// HIP call is made on an error path.  The split of the work over waves and workgroups is a
// function of the sizes alone, so the workspace functions and the calls agree on it.
#include <algorithm>
#include <cmath>

#include "box_relation.h"
#include "evict.hpp"

using namespace rex;

namespace {

size_t align256(size_t x) { return (x + 255) & ~static_cast<size_t>(255); }
bool valid_dtype(int32_t d) { return d == RE_DTYPE_F32 || d == RE_DTYPE_BF16; }
int64_t dtype_size(int32_t d) { return d == RE_DTYPE_BF16 ? 2 : 4; }
bool aligned(const void *p, uintptr_t n) { return reinterpret_cast<uintptr_t>(p) % n == 0; }
re_status_t from_hip(hipError_t e) { return e == hipSuccess ? RE_OK : RE_ERR_DEVICE; }

constexpr int64_t kMaxSpan = kBufMaxBytes - 1;         // bytes of one image's rows
constexpr int64_t kMaxRows = int64_t(1) << 24;         // queries or keys of one image
constexpr int64_t kMaxRowHeads = (int64_t(1) << 31) - 1;
// Workgroups among which the attention's work is shared out: one for each of the 256 CUs, two
// where they have 16 columns, whose few registers leave their waves waiting for memory.  Dense,
// 1000 queries and keys, 16 heads of 64 channels: 128 workgroups 40 us, 256 29.5, 512 42.
// Memory, 300 queries against 6000 boxes in the same heads, the joining of their parts with it: 80 of
// them 90 us, 240 60, 480 73; 64 single queries against up to 8192 boxes each in 8 heads of 32: 256 109,
// 512 83, 1024 93.
constexpr int64_t kGroups = 256;
// Workgroups of the norms.  16000 rows of 1024 channels, bf16: forward 26.6 us with 1024
// of them, 28.2 with 4096; backward 54 us with 512 (two on each CU, what its registers
// allow) and 4 us for their partial sums, 58 us with 1024 and twice the partial sums.
constexpr int64_t kNormBlocks = 1024;
constexpr int64_t kNormSums = 512;
constexpr int64_t kHistTables = 2048;                  // partial tables of the bias gradient

// One side's rows, checked: element strides of batch, row and head, adjacent channels.
re_status_t check_rows(const void *p, int64_t batch, int64_t num, int32_t heads, int32_t dim,
                       const int64_t (&stride)[3], int32_t dtype, Rows *out) {
    const int64_t size = dtype_size(dtype);
    *out = Rows{};
    if (batch == 0 || num == 0) return RE_OK;
    if (!p || !aligned(p, 16)) return RE_ERR_INVALID_ARG;
    int64_t s[3] = {batch > 1 ? stride[0] : 0, num > 1 ? stride[1] : 0, heads > 1 ? stride[2] : 0};
    for (int64_t v : s)
        if (v < 0 || v > (int64_t(1) << 48) || v * size % 16 != 0) return RE_ERR_INVALID_ARG;
    const double span = (double(num + kTile) * double(s[1]) + double(heads - 1) * double(s[2]) + dim) *
                        double(size);
    if (span > double(kMaxSpan) || double(batch) * double(s[0]) > 1e18) return RE_ERR_UNSUPPORTED;
    out->p = p;
    out->sb = s[0] * size;
    out->sr = static_cast<uint32_t>(s[1] * size);
    out->sh = static_cast<uint32_t>(s[2] * size);
    return RE_OK;
}

re_status_t check_shape(int64_t batch, int64_t nq, int64_t nk, int32_t heads, int32_t kv_heads,
                        int32_t dim, int32_t dtype, float scale) {
    if (!valid_dtype(dtype)) return RE_ERR_INVALID_ARG;
    if (batch < 0 || nq < 0 || nk < 0) return RE_ERR_INVALID_ARG;
    if (heads < 1 || kv_heads < 1 || heads > RE_ATTN_MAX_HEADS || heads % kv_heads != 0)
        return RE_ERR_INVALID_ARG;
    if (dim < 8 || dim > RE_ATTN_MAX_DIM || dim % 8 != 0) return RE_ERR_INVALID_ARG;
    if (!std::isfinite(scale) || !(scale >= 1e-20f)) return RE_ERR_INVALID_ARG;
    if (nq > kMaxRows || nk > kMaxRows || batch > kMaxRowHeads) return RE_ERR_UNSUPPORTED;
    if (double(batch) * heads * double(std::max(nq, nk) + kTile) > double(kMaxRowHeads))
        return RE_ERR_UNSUPPORTED;
    // the dense results of one image
    if ((nq + kTile) * heads * dim * dtype_size(dtype) > kMaxSpan) return RE_ERR_UNSUPPORTED;
    return RE_OK;
}

re_status_t check_bias(const float *bias, int32_t buckets, int32_t first_exp, int32_t octave_steps,
                       const float *qbox, const int64_t (&qs)[2], bool need_q, const float *kbox,
                       const int64_t (&ks)[2], bool need_k, BucketRule *rule) {
    *rule = BucketRule{};
    if (!bias) return RE_OK;
    if (buckets < 1 || buckets > RE_ATTN_MAX_BUCKETS || buckets % 2 == 0) return RE_ERR_INVALID_ARG;
    if (first_exp < -64 || first_exp > 64) return RE_ERR_INVALID_ARG;
    if (octave_steps != 1 && octave_steps != 2 && octave_steps != 4) return RE_ERR_INVALID_ARG;
    if (!aligned(bias, 4) || !aligned(qbox, 4) || !aligned(kbox, 4)) return RE_ERR_INVALID_ARG;
    if ((need_q && !qbox) || (need_k && !kbox)) return RE_ERR_INVALID_ARG;
    const int64_t most = int64_t(1) << 48;
    for (int64_t v : {qs[0], qs[1], ks[0], ks[1]})
        if (v < 0 || v > most) return RE_ERR_INVALID_ARG;
    rule->nb = buckets;
    rule->half = (buckets - 1) / 2;
    const int log_steps = octave_steps == 4 ? 2 : octave_steps - 1;
    rule->shift = 23 - log_steps;
    rule->base = (127 + first_exp) * octave_steps;
    return RE_OK;
}

// The largest number of heads, a power of two up to the waves, that a workgroup can take.
int most_heads(int heads, int most) {
    int hp = 1;
    while (hp < most && heads % (2 * hp) == 0) hp *= 2;
    return hp;
}

// Columns of a workgroup: 32, or 16 where there are no more, and for heads of more than 64
// channels, whose sums would fill the registers.
int columns(int64_t rows, int dim) { return rows <= 16 || dim > 64 ? 16 : 32; }

// Heads of a workgroup, whose remaining waves share the streamed tiles, and (`split`) the
// workgroups that share a head's tiles: as many workgroups as there may be, of those choices the
// one with the fewest partial sums.  Heads of one workgroup share the work on buckets, so nothing
// is shared out further than that.
void share_waves(AttnArgs &a, int heads, int64_t blocks, int64_t streamed, int cols, bool split,
                 int most = kAttnWaves) {
    const int64_t groups = kGroups * (cols == 16 ? 2 : 1);
    int64_t best = 0;
    for (int hp = most_heads(heads, most);; hp /= 2) {
        const int parts = kAttnWaves / hp;
        const int64_t wgs = blocks * (heads / hp);
        if (best > 0 && (wgs > groups || parts > streamed)) break;
        // four steps of every wave at least
        const int64_t n = split && wgs > 0 ? std::max<int64_t>(1, std::min(groups / wgs, streamed / (4 * parts))) : 1;
        if (wgs * n >= best) {
            best = wgs * n;
            a.hp = hp;
            a.parts = parts;
            a.nsplit = static_cast<int32_t>(n);
        }
        if (hp == 1) break;
    }
}

// The forward's split, for dense keys and for the memory.
void plan_fwd(AttnArgs &a, int *cols) {
    *cols = columns(a.Nq, a.D);
    a.tiles = (a.Nq + *cols - 1) / *cols;
    const int64_t blocks = static_cast<int64_t>(a.B) * a.tiles;
    share_waves(a, a.H, blocks, (a.Nk + kTile - 1) / kTile, *cols, true);
    a.nwg = static_cast<int32_t>(blocks * (a.H / a.hp) * a.nsplit);
    a.per = a.tiles * a.nsplit;
}

size_t fwd_bytes(const AttnArgs &a) {
    if (a.nsplit <= 1) return 0;
    const size_t rows = static_cast<size_t>(a.nsplit) * a.B * a.H * a.Nq;
    return align256(rows * a.D * 4) + align256(rows * sizeof(SumRef));
}

void place_fwd(AttnArgs &a, void *ws) {
    if (a.nsplit <= 1) return;
    const size_t rows = static_cast<size_t>(a.nsplit) * a.B * a.H * a.Nq;
    a.part = static_cast<float *>(ws);
    a.part_ml = reinterpret_cast<SumRef *>(static_cast<char *>(ws) + align256(rows * a.D * 4));
}

// The backward's two passes.
void plan_bwd(const AttnArgs &a, int dtype, AttnArgs *dq, AttnArgs *dkv, int *dq_cols, int *dkv_cols) {
    *dq = a;
    dq->Nqp = (a.Nq + kTile - 1) / kTile * kTile;
    *dkv = *dq;
    *dq_cols = columns(a.Nq, a.D);
    dq->tiles = dq->per = (a.Nq + *dq_cols - 1) / *dq_cols;
    const int64_t all = static_cast<int64_t>(a.B) * dq->tiles;
    share_waves(*dq, a.H, all, (a.Nk + kTile - 1) / kTile, *dq_cols, false);
    dq->nwg = static_cast<int32_t>(all * (a.H / dq->hp));

    // the heads of a group whose histograms share 64 KiB of LDS
    const int tables = kAttnWaves * std::max(1, a.rule.nb * a.rule.nb) * 8;
    dkv->head_step = std::min({a.group, 4, std::max(1, (64 << 10) / tables)});
    // 16 for binary32 heads of more than 32 channels too, whose operands fill the registers
    // (three images of 171 boxes, six heads of 48: 43 us, 83 with 32)
    *dkv_cols = dtype == RE_DTYPE_F32 && a.D > 32 ? 16 : columns(a.Nk, a.D);
    for (int most = kAttnWaves;;) {
        dkv->tiles = (a.Nk + *dkv_cols - 1) / *dkv_cols;
        const int64_t tiles = static_cast<int64_t>(a.B) * dkv->tiles;
        dkv->span = static_cast<int32_t>(std::max<int64_t>(1, a.bias ? (tiles + kHistTables - 1) / kHistTables : 1));
        dkv->spans = dkv->per = (dkv->tiles + dkv->span - 1) / dkv->span;
        const int64_t blocks = static_cast<int64_t>(a.B) * dkv->spans;
        share_waves(*dkv, a.Hkv, blocks, (a.Nq + kTile - 1) / kTile, *dkv_cols, false, most);
        dkv->nwg = static_cast<int32_t>(blocks * (a.Hkv / dkv->hp));
        // beside the largest tables there is room for 16 columns only, or for fewer heads
        if (dkv_fits(*dkv, dtype, *dkv_cols)) break;
        if (*dkv_cols > 16) *dkv_cols = 16;
        else most = dkv->hp / 2;
    }
}

size_t stat_bytes(const AttnArgs &dq) {          // of rowstat, and of rowfar
    return align256(static_cast<size_t>(dq.B) * dq.H * dq.Nqp * 8);
}
size_t far_bytes(const AttnArgs &dq) { return align256(static_cast<size_t>(dq.B) * dq.H * dq.Nqp / 4); }
size_t bwd_bytes(const AttnArgs &dkv) {
    const size_t nb2 = static_cast<size_t>(dkv.rule.nb) * dkv.rule.nb;
    return 2 * stat_bytes(dkv) + far_bytes(dkv) + (dkv.bias ? align256(static_cast<size_t>(dkv.B) * dkv.spans * dkv.H * nb2 * 4) : 0);
}

re_status_t attn_args(const box_attn_t *d, AttnArgs *a) {
    *a = AttnArgs{};
    if (!d) return RE_ERR_INVALID_ARG;
    re_status_t st = check_shape(d->batch, d->num_q, d->num_k, d->heads, d->kv_heads, d->dim,
                                 d->dtype, d->scale);
    if (st != RE_OK) return st;
    if ((d->num_k + kTile) * d->kv_heads * d->dim * dtype_size(d->dtype) > kMaxSpan) return RE_ERR_UNSUPPORTED;
    if ((st = check_rows(d->q, d->batch, d->num_q, d->heads, d->dim, d->q_stride, d->dtype, &a->q)) != RE_OK)
        return st;
    if ((st = check_rows(d->k, d->batch, d->num_k, d->kv_heads, d->dim, d->k_stride, d->dtype, &a->k)) != RE_OK)
        return st;
    if ((st = check_rows(d->v, d->batch, d->num_k, d->kv_heads, d->dim, d->v_stride, d->dtype, &a->v)) != RE_OK)
        return st;
    if ((st = check_bias(d->bias, d->buckets, d->first_exp, d->octave_steps, d->q_boxes,
                         d->q_box_stride, d->batch * d->num_q > 0, d->k_boxes, d->k_box_stride,
                         d->batch * d->num_k > 0, &a->rule)) != RE_OK)
        return st;
    if (!d->bias && d->buckets != 0) return RE_ERR_INVALID_ARG;
    if (!aligned(d->q_len, 4) || !aligned(d->k_len, 4)) return RE_ERR_INVALID_ARG;
    a->qbox = d->q_boxes;
    a->kbox = d->k_boxes;
    if (d->bias) {
        a->qbox_sb = d->q_box_stride[0];
        a->qbox_sr = d->q_box_stride[1];
        a->kbox_sb = d->k_box_stride[0];
        a->kbox_sr = d->k_box_stride[1];
    }
    a->bias = d->bias;
    a->qlen = d->q_len;
    a->klen = d->k_len;
    a->kmask = d->k_mask;
    a->scale = d->scale;
    a->B = static_cast<int32_t>(d->batch);
    a->Nq = static_cast<int32_t>(d->num_q);
    a->Nk = static_cast<int32_t>(d->num_k);
    a->H = d->heads;
    a->Hkv = d->kv_heads;
    a->D = d->dim;
    a->group = d->heads / d->kv_heads;
    return RE_OK;
}

re_status_t check_workspace(const void *ws, size_t have, size_t need) {
    if (need == 0) return RE_OK;
    if (!ws || have < need || !aligned(ws, 256)) return RE_ERR_WORKSPACE;
    return RE_OK;
}

}  // namespace

namespace rex {
re_status_t check_memory(const box_memory_t *m) {
    if (!m || !m->k || !m->v || !m->k_scale || !m->v_scale || !m->boxes) return RE_ERR_INVALID_ARG;
    if (!aligned(m->k, 16) || !aligned(m->v, 16) || !aligned(m->k_scale, 16) ||
        !aligned(m->v_scale, 16) || !aligned(m->boxes, 16))
        return RE_ERR_INVALID_ARG;
    if (m->num_pages < 1 || m->num_pages > INT32_MAX) return RE_ERR_INVALID_ARG;
    if (m->kv_heads < 1 || m->kv_heads > RE_ATTN_MAX_HEADS) return RE_ERR_INVALID_ARG;
    if (m->dim < 8 || m->dim > RE_ATTN_MAX_DIM || m->dim % 8 != 0) return RE_ERR_INVALID_ARG;
    return RE_OK;
}

re_status_t recall_args(const box_memory_t *m, const box_recall_t *r, AttnArgs *a) {
    *a = AttnArgs{};
    re_status_t st = check_memory(m);
    if (st != RE_OK) return st;
    if (!r) return RE_ERR_INVALID_ARG;
    if (r->max_pages < 0) return RE_ERR_INVALID_ARG;
    if (r->max_pages > kMaxRows / kTile) return RE_ERR_UNSUPPORTED;
    if ((st = check_shape(r->batch, r->num_q, r->max_pages * kTile, r->heads, m->kv_heads, m->dim,
                          r->dtype, r->scale)) != RE_OK)
        return st;
    if ((st = check_rows(r->q, r->batch, r->num_q, r->heads, m->dim, r->q_stride, r->dtype, &a->q)) != RE_OK)
        return st;
    if ((st = check_bias(r->bias, r->buckets, r->first_exp, r->octave_steps, r->q_boxes,
                         r->q_box_stride, r->batch * r->num_q > 0, nullptr, r->q_box_stride, false,
                         &a->rule)) != RE_OK)
        return st;
    if (!r->bias && r->buckets != 0) return RE_ERR_INVALID_ARG;
    if (r->batch > 0 && (!r->lengths || (r->max_pages > 0 && !r->pages))) return RE_ERR_INVALID_ARG;
    if (!aligned(r->lengths, 4) || !aligned(r->pages, 4) || !aligned(r->q_len, 4))
        return RE_ERR_INVALID_ARG;
    a->qbox = r->q_boxes;
    if (r->bias) {
        a->qbox_sb = r->q_box_stride[0];
        a->qbox_sr = r->q_box_stride[1];
    }
    a->bias = r->bias;
    a->qlen = r->q_len;
    a->klen = r->lengths;
    a->scale = r->scale;
    a->B = static_cast<int32_t>(r->batch);
    a->Nq = static_cast<int32_t>(r->num_q);
    a->Nk = static_cast<int32_t>(r->max_pages * kTile);
    a->H = r->heads;
    a->Hkv = m->kv_heads;
    a->D = m->dim;
    a->group = r->heads / m->kv_heads;
    a->mk = m->k;
    a->mv = m->v;
    a->mks = m->k_scale;
    a->mvs = m->v_scale;
    a->mbox = m->boxes;
    a->pages = r->pages;
    a->num_pages = m->num_pages;
    a->max_pages = static_cast<int32_t>(r->max_pages);
    return RE_OK;
}
}  // namespace rex

namespace {

// The norm's arguments and the shares of the backward's workgroups.
re_status_t norm_args(const gated_norm_t *d, NormArgs *a) {
    *a = NormArgs{};
    if (!d) return RE_ERR_INVALID_ARG;
    if (!valid_dtype(d->dtype)) return RE_ERR_INVALID_ARG;
    if (d->norm != RE_NORM_RMS && d->norm != RE_NORM_LAYER) return RE_ERR_INVALID_ARG;
    if (d->rows < 0 || d->channels < 1 || d->gates < 0) return RE_ERR_INVALID_ARG;
    if (d->rows > kMaxRowHeads || d->channels > RE_NORM_MAX_CHANNELS) return RE_ERR_UNSUPPORTED;
    if (!std::isfinite(d->alpha) || !std::isfinite(d->eps) || !(d->eps > 0.0f)) return RE_ERR_INVALID_ARG;
    const uintptr_t size = static_cast<uintptr_t>(dtype_size(d->dtype));
    if (d->rows > 0 && !d->x) return RE_ERR_INVALID_ARG;
    if (!aligned(d->x, size) || !aligned(d->branch, size)) return RE_ERR_INVALID_ARG;
    const int64_t most = int64_t(1) << 31;
    if (d->rows > 1 && (d->x_stride < 0 || d->x_stride > most)) return RE_ERR_INVALID_ARG;
    if (d->rows > 1 && d->branch && (d->branch_stride < 0 || d->branch_stride > most))
        return RE_ERR_INVALID_ARG;
    if ((d->gate != nullptr) != (d->gates > 0)) return RE_ERR_INVALID_ARG;
    if (d->gate && (d->rows % d->gates != 0 || (d->rows > 0 && !d->branch))) return RE_ERR_INVALID_ARG;
    for (const float *p : {d->gate, d->post_weight, d->post_bias, d->pre_weight, d->pre_bias})
        if (!aligned(p, 4)) return RE_ERR_INVALID_ARG;
    a->x = d->x;
    a->branch = d->branch;
    a->x_stride = d->rows > 1 ? d->x_stride : 0;
    a->b_stride = d->rows > 1 ? d->branch_stride : 0;
    a->rows = d->rows;
    a->gates = d->gates;
    a->rows_per_gate = d->gates > 0 ? std::max<int64_t>(1, d->rows / d->gates) : 1;
    a->C = d->channels;
    a->layer = d->norm == RE_NORM_LAYER;
    a->alpha = d->alpha;
    a->eps = d->eps;
    a->gate = d->gate;
    a->w1 = d->post_weight;
    a->c1 = d->post_bias;
    a->w2 = d->pre_weight;
    a->c2 = d->pre_bias;
    const int64_t chunk = 16 / static_cast<int64_t>(size);
    a->vec = d->channels % chunk == 0 && aligned(d->x, 16) && aligned(d->branch, 16) &&
             a->x_stride % chunk == 0 && a->b_stride % chunk == 0;
    a->gate_div = make_fastdiv(static_cast<uint32_t>(std::max<int64_t>(1, a->rows_per_gate)));
    a->pvec = d->channels % 4 == 0 && aligned(d->gate, 16) && aligned(d->post_weight, 16) &&
              aligned(d->post_bias, 16) && aligned(d->pre_weight, 16) && aligned(d->pre_bias, 16);
    // units of the backward: runs of rows of one gate row
    const int slots = norm_slots(d->dtype, a->C);
    const bool each = !d->gate || a->rows_per_gate == 1;
    a->span = each ? a->rows : a->rows_per_gate;
    const int64_t segments = a->rows == 0 ? 0 : each ? 1 : d->gates;
    if (segments > 0) {
        const int64_t parts = std::min((kNormSums + segments - 1) / segments, (a->span + slots - 1) / slots);
        a->gate_parts = static_cast<int32_t>(parts);
        a->unit_rows = static_cast<int32_t>((a->span + parts - 1) / parts);
        a->units = segments * parts;
    }
    a->blocks = static_cast<int32_t>(std::min<int64_t>(a->units, kNormSums));
    return RE_OK;
}

size_t norm_part_bytes(const NormArgs &a) { return align256(static_cast<size_t>(a.blocks) * 4 * a.C * 4); }
size_t norm_bytes(const NormArgs &a) {
    const bool shared = a.gate && a.rows_per_gate > 1;
    return norm_part_bytes(a) + (shared ? align256(static_cast<size_t>(a.units) * a.C * 4) : 0);
}

}  // namespace

extern "C" {

re_status_t box_attn_workspace_size(const box_attn_t *d, int32_t backward, size_t *bytes) {
    if (!bytes) return RE_ERR_INVALID_ARG;
    AttnArgs a, dq, dkv;
    int c0, c1;
    const re_status_t st = attn_args(d, &a);
    if (st != RE_OK) return st;
    plan_fwd(a, &c0);
    *bytes = fwd_bytes(a);
    if (backward) {
        plan_bwd(a, d->dtype, &dq, &dkv, &c0, &c1);
        *bytes = std::max(*bytes, bwd_bytes(dkv));
    }
    return RE_OK;
}

re_status_t box_attn_fwd(const box_attn_t *d, void *out, float *lse, float *out_f32,
                         void *workspace, size_t workspace_bytes, void *stream) {
    AttnArgs a;
    int cols = 0;
    re_status_t st = attn_args(d, &a);
    if (st != RE_OK) return st;
    if (a.B == 0 || a.Nq == 0) return RE_OK;
    if (!out || !aligned(out, 16) || !aligned(lse, 4) || !aligned(out_f32, 16)) return RE_ERR_INVALID_ARG;
    plan_fwd(a, &cols);
    if ((st = check_workspace(workspace, workspace_bytes, fwd_bytes(a))) != RE_OK) return st;
    place_fwd(a, workspace);
    a.out = out;
    a.lse = lse;
    a.out_f32 = out_f32;
    // out_f32 is what the backward subtracts from the logits' gradient: with few keys that may leave
    // nothing (with one key it does), so all bits of the weights count
    a.terms = out_f32 && a.Nk <= RE_ATTN_FEW_KEYS ? 3 : 2;
    const hipStream_t s = static_cast<hipStream_t>(stream);
    if ((st = from_hip(launch_attn_fwd(a, d->dtype, cols, s))) != RE_OK || a.nsplit == 1) return st;
    return from_hip(launch_attn_combine(a, d->dtype, s));
}

re_status_t box_attn_bwd(const box_attn_t *d, const void *grad_out, const void *out,
                         const float *lse, const float *out_f32, void *grad_q, void *grad_k,
                         void *grad_v, float *grad_bias, void *workspace, size_t workspace_bytes,
                         void *stream) {
    AttnArgs a, dq, dkv;
    int c0 = 0, c1 = 0;
    re_status_t st = attn_args(d, &a);
    if (st != RE_OK) return st;
    const bool rows = a.B > 0 && a.Nq > 0, keys = a.B > 0 && a.Nk > 0;
    if (rows && (!grad_out || !out || !lse || !grad_q)) return RE_ERR_INVALID_ARG;
    if (keys && (!grad_k || !grad_v)) return RE_ERR_INVALID_ARG;
    if ((grad_bias != nullptr) != (d->bias != nullptr)) return RE_ERR_INVALID_ARG;
    for (const void *p : {grad_out, out, static_cast<const void *>(out_f32), static_cast<const void *>(grad_q),
                          static_cast<const void *>(grad_k), static_cast<const void *>(grad_v)})
        if (!aligned(p, 16)) return RE_ERR_INVALID_ARG;
    if (!aligned(lse, 4) || !aligned(grad_bias, 4)) return RE_ERR_INVALID_ARG;
    const int64_t size = dtype_size(d->dtype), row = static_cast<int64_t>(a.H) * a.D * size;
    a.gout = Rows{grad_out, a.Nq * row, static_cast<uint32_t>(row), static_cast<uint32_t>(a.D * size)};
    a.fout = out;
    a.fout_f32 = out_f32;
    a.flse = lse;
    a.gq = grad_q;
    a.gk = grad_k;
    a.gv = grad_v;
    a.gbias = grad_bias;
    plan_bwd(a, d->dtype, &dq, &dkv, &c0, &c1);
    if ((st = check_workspace(workspace, workspace_bytes, bwd_bytes(dkv))) != RE_OK) return st;
    char *ws = static_cast<char *>(workspace);
    dq.rowstat = dkv.rowstat = reinterpret_cast<float *>(ws);
    dq.rowfar = dkv.rowfar = reinterpret_cast<float *>(ws += stat_bytes(dkv));
    dq.far = dkv.far = reinterpret_cast<int32_t *>(ws += stat_bytes(dkv));
    dkv.hist = reinterpret_cast<float *>(ws + far_bytes(dkv));
    return from_hip(launch_attn_bwd(dq, dkv, d->dtype, c0, c1, static_cast<hipStream_t>(stream)));
}

re_status_t box_memory_append(const box_memory_t *m, const int64_t *slots, int64_t count,
                              const void *k, const void *v, int32_t dtype,
                              const int64_t k_stride[2], const int64_t v_stride[2],
                              const float *boxes, void *stream) {
    const re_status_t st = check_memory(m);
    if (st != RE_OK) return st;
    if (!valid_dtype(dtype) || count < 0) return RE_ERR_INVALID_ARG;
    if (count > kMaxRowHeads / RE_ATTN_MAX_HEADS) return RE_ERR_UNSUPPORTED;
    if (count == 0) return RE_OK;
    const uintptr_t size = static_cast<uintptr_t>(dtype_size(dtype));
    if (!slots || !k || !v || !boxes || !k_stride || !v_stride) return RE_ERR_INVALID_ARG;
    if (!aligned(slots, 8) || !aligned(k, size) || !aligned(v, size) || !aligned(boxes, 4))
        return RE_ERR_INVALID_ARG;
    MemoryArgs a{};
    const int64_t chunk = 16 / static_cast<int64_t>(size), most = int64_t(1) << 31;
    a.vec = aligned(k, 16) && aligned(v, 16);
    for (int64_t s : {k_stride[0], k_stride[1], v_stride[0], v_stride[1]}) {
        if (s < 0 || s > most) return RE_ERR_INVALID_ARG;
        a.vec = a.vec && s % chunk == 0;
    }
    a.k8 = m->k;
    a.v8 = m->v;
    a.ks = m->k_scale;
    a.vs = m->v_scale;
    a.mbox = m->boxes;
    a.num_slots = m->num_pages * kTile;
    a.Hkv = m->kv_heads;
    a.D = m->dim;
    a.slots = slots;
    a.count = count;
    a.k = k;
    a.v = v;
    a.k_sr = k_stride[0];
    a.k_sh = k_stride[1];
    a.v_sr = v_stride[0];
    a.v_sh = v_stride[1];
    a.boxes = boxes;
    return from_hip(launch_memory_append(a, dtype, static_cast<hipStream_t>(stream)));
}

re_status_t box_memory_read(const box_memory_t *m, const int64_t *slots, int64_t count, void *k_out,
                            void *v_out, int32_t dtype, float *boxes_out, void *stream) {
    const re_status_t st = check_memory(m);
    if (st != RE_OK) return st;
    if (!valid_dtype(dtype) || count < 0) return RE_ERR_INVALID_ARG;
    if (count > kMaxRowHeads / RE_ATTN_MAX_HEADS) return RE_ERR_UNSUPPORTED;
    if (count == 0) return RE_OK;
    if (!slots || !aligned(slots, 8)) return RE_ERR_INVALID_ARG;
    if (!aligned(k_out, 16) || !aligned(v_out, 16) || !aligned(boxes_out, 4)) return RE_ERR_INVALID_ARG;
    MemoryArgs a{};
    a.k8 = m->k;
    a.v8 = m->v;
    a.ks = m->k_scale;
    a.vs = m->v_scale;
    a.mbox = m->boxes;
    a.num_slots = m->num_pages * kTile;
    a.Hkv = m->kv_heads;
    a.D = m->dim;
    a.slots = slots;
    a.count = count;
    a.k_out = k_out;
    a.v_out = v_out;
    a.boxes_out = boxes_out;
    return from_hip(launch_memory_read(a, dtype, static_cast<hipStream_t>(stream)));
}

re_status_t box_memory_attn_workspace_size(const box_memory_t *m, const box_recall_t *r, size_t *bytes) {
    if (!bytes) return RE_ERR_INVALID_ARG;
    AttnArgs a;
    int cols;
    const re_status_t st = recall_args(m, r, &a);
    if (st != RE_OK) return st;
    plan_fwd(a, &cols);
    *bytes = fwd_bytes(a);
    return RE_OK;
}

re_status_t box_memory_attn_fwd(const box_memory_t *m, const box_recall_t *r, void *out, float *lse,
                                void *workspace, size_t workspace_bytes, void *stream) {
    AttnArgs a;
    int cols = 0;
    re_status_t st = recall_args(m, r, &a);
    if (st != RE_OK) return st;
    if (a.B == 0 || a.Nq == 0) return RE_OK;
    if (!out || !aligned(out, 16) || !aligned(lse, 4)) return RE_ERR_INVALID_ARG;
    plan_fwd(a, &cols);
    if ((st = check_workspace(workspace, workspace_bytes, fwd_bytes(a))) != RE_OK) return st;
    place_fwd(a, workspace);
    a.out = out;
    a.lse = lse;
    const hipStream_t s = static_cast<hipStream_t>(stream);
    if ((st = from_hip(launch_attn_recall(a, r->dtype, cols, s))) != RE_OK || a.nsplit == 1) return st;
    return from_hip(launch_attn_combine(a, r->dtype, s));
}

re_status_t gated_norm_fwd(const gated_norm_t *d, void *y, void *u, float *stats, void *stream) {
    NormArgs a;
    const re_status_t st = norm_args(d, &a);
    if (st != RE_OK) return st;
    const uintptr_t size = static_cast<uintptr_t>(dtype_size(d->dtype));
    if (a.rows == 0) return RE_OK;
    if (!y && (!u || d->branch)) return RE_ERR_INVALID_ARG;
    if (!aligned(y, size) || !aligned(u, size) || !aligned(stats, 16)) return RE_ERR_INVALID_ARG;
    a.y = y;
    a.u = u;
    a.stats = stats;
    a.second = u != nullptr;
    a.vec = a.vec && aligned(y, 16) && aligned(u, 16);
    // rows in runs, as many workgroups as fill the GPU several times over
    const int64_t slots = norm_slots(d->dtype, a.C), groups = (a.rows + slots - 1) / slots;
    a.unit_rows = static_cast<int32_t>((groups + kNormBlocks - 1) / kNormBlocks * slots);
    a.blocks = static_cast<int32_t>((a.rows + a.unit_rows - 1) / a.unit_rows);
    return from_hip(launch_norm_fwd(a, d->dtype, static_cast<hipStream_t>(stream)));
}

re_status_t gated_norm_workspace_size(const gated_norm_t *d, size_t *bytes) {
    if (!bytes) return RE_ERR_INVALID_ARG;
    NormArgs a;
    const re_status_t st = norm_args(d, &a);
    if (st != RE_OK) return st;
    *bytes = norm_bytes(a);
    return RE_OK;
}

re_status_t gated_norm_bwd(const gated_norm_t *d, const void *grad_y, const void *grad_u,
                           const float *stats, const gated_norm_grads_t *grads, void *workspace,
                           size_t workspace_bytes, void *stream) {
    NormArgs a;
    re_status_t st = norm_args(d, &a);
    if (st != RE_OK) return st;
    if (!grads) return RE_ERR_INVALID_ARG;
    const uintptr_t size = static_cast<uintptr_t>(dtype_size(d->dtype));
    if (a.rows > 0 && (!stats || !aligned(stats, 16))) return RE_ERR_INVALID_ARG;
    for (const void *p : {grad_y, grad_u, static_cast<const void *>(grads->x),
                          static_cast<const void *>(grads->branch)})
        if (!aligned(p, size)) return RE_ERR_INVALID_ARG;
    for (const float *p : {grads->gate, grads->post_weight, grads->post_bias, grads->pre_weight,
                           grads->pre_bias})
        if (!aligned(p, 4)) return RE_ERR_INVALID_ARG;
    if (a.rows > 0 && !d->branch && (grads->branch || grads->gate || grads->post_weight || grads->post_bias))
        return RE_ERR_INVALID_ARG;
    if (grads->gate && !d->gate) return RE_ERR_INVALID_ARG;
    if ((st = check_workspace(workspace, workspace_bytes, norm_bytes(a))) != RE_OK) return st;
    a.gy = grad_y;
    a.gu = grad_u;
    a.stats = const_cast<float *>(stats);
    a.gx = grads->x;
    a.gb = grads->branch;
    a.ggate = grads->gate;
    a.gw1 = grads->post_weight;
    a.gc1 = grads->post_bias;
    a.gw2 = grads->pre_weight;
    a.gc2 = grads->pre_bias;
    a.vec = a.vec && aligned(grad_y, 16) && aligned(grad_u, 16) && aligned(a.gx, 16) && aligned(a.gb, 16);
    a.part = static_cast<float *>(workspace);
    // a gate that several rows share is summed in parts
    a.gate_sum = a.ggate && (a.rows_per_gate > 1 || a.rows == 0);
    if (a.gate_sum && a.units > 0)
        a.gate_part = reinterpret_cast<float *>(static_cast<char *>(workspace) + norm_part_bytes(a));
    return from_hip(launch_norm_bwd(a, d->dtype, static_cast<hipStream_t>(stream)));
}

}  // extern "C"
