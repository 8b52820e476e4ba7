// evict_api.hip -- the C ABI declared in include/box_evict.h.
//
// As in api.hip, every argument is checked on the host before anything is enqueued, and no
// HIP call is made on an error path.
#include <cmath>

#include "evict.hpp"

using namespace rex;

namespace {

constexpr int64_t kMaxPlaces = int64_t(1) << 24;       // of one stream
size_t align256(size_t x) { return (x + 255) & ~static_cast<size_t>(255); }
bool aligned(const void *p, uintptr_t n) { return reinterpret_cast<uintptr_t>(p) % n == 0; }
re_status_t from_hip(hipError_t e) { return e == hipSuccess ? RE_OK : RE_ERR_DEVICE; }

re_status_t check_workspace(const void *ws, size_t have, size_t need) {
    if (need == 0) return RE_OK;
    if (!ws || have < need || !aligned(ws, 256)) return RE_ERR_WORKSPACE;
    return RE_OK;
}

re_status_t evict_args(const box_memory_t *m, const box_evict_t *d, EvictArgs *e) {
    *e = EvictArgs{};
    const re_status_t st = check_memory(m);
    if (st != RE_OK) return st;
    if (!d || d->batch < 0 || d->max_pages < 0) return RE_ERR_INVALID_ARG;
    if (d->max_pages > kMaxPlaces / kTile || d->batch > (1 << 21)) return RE_ERR_UNSUPPORTED;
    // a launch has fewer than 2^32 threads: 256 for every page and four key heads
    if (double(d->batch) * double(d->max_pages) * ((m->kv_heads + 3) / 4) >= double(1 << 24)) return RE_ERR_UNSUPPORTED;
    if (d->batch > 0 && (!d->lengths || !d->keep || (d->max_pages > 0 && (!d->pages || !d->weight)))) return RE_ERR_INVALID_ARG;
    if (!aligned(d->pages, 4) || !aligned(d->lengths, 4) || !aligned(d->keep, 4) || !aligned(d->weight, 4))
        return RE_ERR_INVALID_ARG;
    e->k = m->k;
    e->v = m->v;
    e->ks = m->k_scale;
    e->vs = m->v_scale;
    e->boxes = m->boxes;
    e->num_pages = m->num_pages;
    e->Hkv = m->kv_heads;
    e->D = m->dim;
    e->B = static_cast<int32_t>(d->batch);
    e->max_pages = static_cast<int32_t>(d->max_pages);
    e->pages = d->pages;
    e->lengths = d->lengths;
    e->keep = d->keep;
    e->weight = d->weight;
    return RE_OK;
}
size_t evict_part_bytes(const EvictArgs &e) { return align256(static_cast<size_t>(e.B) * e.max_pages * kTile * 4); }

}  // namespace

extern "C" {

re_status_t box_memory_weigh(const box_memory_t *m, const box_recall_t *r, const float *lse,
                             const float *weight, float decay, float *weight_out, void *stream) {
    WeighArgs w{};
    const re_status_t st = recall_args(m, r, &w.a);
    if (st != RE_OK) return st;
    if (weight && !std::isfinite(decay)) return RE_ERR_INVALID_ARG;
    if (!aligned(lse, 4) || !aligned(weight, 4) || !aligned(weight_out, 4)) return RE_ERR_INVALID_ARG;
    if (w.a.B == 0 || w.a.max_pages == 0) return RE_OK;
    if (!weight_out || (w.a.Nq > 0 && !lse)) return RE_ERR_INVALID_ARG;
    // a launch has fewer than 2^32 threads: a workgroup of 1024 for every page
    if (double(w.a.B) * double(w.a.max_pages) >= double(1 << 22)) return RE_ERR_UNSUPPORTED;
    w.lse = lse;
    w.weight = weight;
    w.decay = decay;
    w.out = weight_out;
    return from_hip(launch_weigh(w, r->dtype, static_cast<hipStream_t>(stream)));
}

re_status_t box_memory_evict_workspace_size(const box_memory_t *m, const box_evict_t *d, size_t *bytes) {
    if (!bytes) return RE_ERR_INVALID_ARG;
    EvictArgs e;
    const re_status_t st = evict_args(m, d, &e);
    if (st != RE_OK) return st;
    *bytes = 4 * evict_part_bytes(e);
    return RE_OK;
}

re_status_t box_memory_evict(const box_memory_t *m, const box_evict_t *d, int32_t *lengths_out,
                             float *weight_out, int32_t *origin, void *workspace,
                             size_t workspace_bytes, void *stream) {
    EvictArgs e;
    re_status_t st = evict_args(m, d, &e);
    if (st != RE_OK) return st;
    if (!aligned(lengths_out, 4) || !aligned(weight_out, 4) || !aligned(origin, 4)) return RE_ERR_INVALID_ARG;
    if (e.B == 0) return RE_OK;
    if (!lengths_out || (e.max_pages > 0 && !weight_out)) return RE_ERR_INVALID_ARG;
    if (weight_out && weight_out == d->weight) return RE_ERR_INVALID_ARG;
    if ((st = check_workspace(workspace, workspace_bytes, 4 * evict_part_bytes(e))) != RE_OK) return st;
    e.lengths_out = lengths_out;
    e.weight_out = weight_out;
    char *ws = static_cast<char *>(workspace);
    e.freed = reinterpret_cast<int32_t *>(ws);
    e.late = reinterpret_cast<int32_t *>(ws + evict_part_bytes(e));
    e.source = reinterpret_cast<int32_t *>(ws + 2 * evict_part_bytes(e));
    e.from = origin ? origin : reinterpret_cast<int32_t *>(ws + 3 * evict_part_bytes(e));
    return from_hip(launch_evict(e, static_cast<hipStream_t>(stream)));
}

}  // extern "C"
