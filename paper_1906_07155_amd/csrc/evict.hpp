// evict.hpp -- argument blocks and launchers of what the memory of boxes forgets.
#pragma once

#include "box_evict.h"
#include "relation.hpp"

namespace rex {

// Of the memory and of a call that reads it (relation_api.hip).
re_status_t check_memory(const box_memory_t *m);
re_status_t recall_args(const box_memory_t *m, const box_recall_t *r, AttnArgs *a);

struct WeighArgs {
    AttnArgs a;                     // the recall's
    const float *lse, *weight;      // weight may be null
    float *out;
    float decay;
};
constexpr int kFewQueries = 16;     // of a stream: one column tile of the products
hipError_t launch_weigh(const WeighArgs &w, int dtype, hipStream_t s);

struct EvictArgs {
    int8_t *k, *v;
    float *ks, *vs, *boxes;
    int64_t num_pages;
    int32_t Hkv, D, B, max_pages;
    const int32_t *pages, *lengths, *keep;
    const float *weight;
    int32_t *lengths_out;
    float *weight_out;
    int32_t *from;                  // [B][places]: the place that a place's box was in, or -1
    int32_t *source;                // [B][places]: the page of that place, where a box moves, else -1
    int32_t *freed, *late;          // [B][places]: of long streams, free places and the boxes that fill them
};
hipError_t launch_evict(const EvictArgs &e, hipStream_t s);

}  // namespace rex
