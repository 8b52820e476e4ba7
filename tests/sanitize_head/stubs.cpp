// Launchers for the host build of head_api.hip and evict_api.hip: they look at every argument and do nothing.
#include "hip/hip_runtime.h"
#include "evict.hpp"
#include "linear.hpp"
#include "logprob.hpp"

#include <cstdio>
#include <cstdlib>

namespace rex {

#define need(ok)                                                      \
    do {                                                              \
        if (!(ok)) {                                                  \
            std::fprintf(stderr, "line %d: %s\n", __LINE__, #ok);     \
            std::abort();                                             \
        }                                                             \
    } while (0)

static bool small(int64_t groups, int threads) { return groups >= 1 && groups * threads < int64_t(1) << 32; }

static hipError_t tiles(const GemmArgs &a, const GemmPlan &p, bool f32) {
    need(a.p && a.q && a.out && a.M >= 1 && a.N >= 1 && a.K >= 1);
    need(p.tile == kTileSmall || p.tile == kTileMiddle || (p.tile == kTileLarge && !f32));
    need(p.chunks || (f32 ? p.tile == kTileSmall : p.tile != kTileLarge));
    need(p.tile == kTileSmall ? p.bm == 64 && p.bn == 64 : p.tile == kTileLarge ? p.bm == 256 && p.bn == 256
                                                                                 : p.bm == 128 && p.bn == (f32 ? 64 : 128));
    need(a.tiles_m == (a.M + p.bm - 1) / p.bm && a.tiles_n == (a.N + p.bn - 1) / p.bn);
    need(int64_t(a.tiles_m) * a.tiles_n == int64_t(a.whole) + a.parted);
    need(a.grid_whole >= a.whole && a.grid_whole < a.whole + 8 && a.grid_whole % 8 == 0);
    need((a.split > 1) == (a.parted > 0) && (a.split == 1 || a.part));
    // the parts cover the sums, none of them empty
    const int64_t steps = (a.K + (f32 ? 31 : 63)) / (f32 ? 32 : 64);
    need(int64_t(a.split) * a.steps >= steps && (int64_t(a.split) - 1) * a.steps < steps);
    need(small(a.grid_whole + int64_t(a.parted) * a.split, p.tile == kTileLarge ? 512 : 256));
    need(!a.vec || a.N % 4 == 0);
    return hipSuccess;
}
hipError_t launch_gemm_bf16(const GemmArgs &a, const GemmPlan &p, bool, bool, hipStream_t) { return tiles(a, p, false); }
hipError_t launch_gemm_f32(const GemmArgs &a, const GemmPlan &p, bool, bool, hipStream_t) { return tiles(a, p, true); }
hipError_t launch_gemm_join(const GemmArgs &a, const GemmPlan &p, int, hipStream_t) {
    need(a.split > 1 && small(int64_t(a.parted) * (p.bm * p.bn / 1024), 256));
    return hipSuccess;
}
hipError_t launch_skinny(const GemmArgs &a, int, bool turned, hipStream_t) {
    const int many = turned ? a.M : a.N, few = turned ? a.N : a.M;
    need(a.p && a.q && a.out && few >= 1 && few <= kSkinnyRows && a.K % 8 == 0 && !(turned && a.vec));
    need(small((int64_t(many) + 15) / 16 * a.split, 1024) && (a.split == 1 || a.part));
    need(int64_t(a.split) * a.steps * 32 >= a.K && (int64_t(a.split) - 1) * a.steps * 32 < a.K);
    return hipSuccess;
}
hipError_t launch_skinny_join(const GemmArgs &a, int, hipStream_t) {
    need(a.split > 1 && small(int64_t(a.M) * ((a.N + 3) / 4) / 256 + 1, 256));
    return hipSuccess;
}
hipError_t launch_slope(const SlopeArgs &a, int, hipStream_t) {
    need(a.blocks == 0 ? a.M == 0 : int64_t(a.blocks) * a.run >= a.M && int64_t(a.blocks - 1) * a.run < a.M);
    need((a.M == 0 || a.gy) && (!a.saved || a.g) && (!a.gbias || a.part || a.blocks == 0));
    need(small((int64_t(a.N) + 63) / 64 * std::max(a.blocks, 1), 256));
    return hipSuccess;
}
hipError_t launch_clear(void *p, int64_t bytes, hipStream_t) {
    need(p && bytes > 0 && bytes % 2 == 0);
    return hipSuccess;
}
static hipError_t logprob(const LogprobArgs &a) {
    need(a.rows >= 1 && a.C >= 1 && a.logits && a.labels && a.stats && a.entropy);
    need(a.each % 8 == 0 || a.parts == 1);
    need(a.each <= kLogprobSpan && int64_t(a.parts) * a.each >= a.C && int64_t(a.parts - 1) * a.each < a.C);
    need(small(a.rows * a.parts, 256));
    return hipSuccess;
}
hipError_t launch_logprob_fwd(const LogprobArgs &a, int, hipStream_t) {
    need(a.logp && (a.parts == 1 || a.part) && (a.top == 0 || (a.top_logp && a.top_index)));
    return logprob(a);
}
hipError_t launch_logprob_bwd(const LogprobArgs &a, int, hipStream_t) {
    need(a.grad);
    return logprob(a);
}
hipError_t launch_weigh(const WeighArgs &w, int, hipStream_t) {
    need(w.out && (w.a.Nq == 0 || w.lse) && small(int64_t(w.a.B) * w.a.max_pages, 1024));
    return hipSuccess;
}
hipError_t launch_evict(const EvictArgs &e, hipStream_t) {
    need(e.B >= 1 && e.lengths_out && small(e.B, 1024));
    need(e.max_pages == 0 ||
         (e.freed && e.late && e.source && e.from && small(int64_t(e.B) * e.max_pages * ((e.Hkv + 3) / 4), 256)));
    return hipSuccess;
}

}  // namespace rex
