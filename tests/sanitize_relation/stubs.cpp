// Launchers for the host build of relation_api.hip: they look at every argument and do nothing.
#include "hip/hip_runtime.h"
#include "relation.hpp"

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
// What the attention's kernels take for granted of their shares.
static void shares(const AttnArgs &a, int heads) {
    need(a.hp >= 1 && a.parts >= 1 && a.hp * a.parts == kAttnWaves && heads % a.hp == 0);
    need(a.nwg == 0 || (a.nwg > 0 && a.per >= 1 && a.tiles >= 1));
}
hipError_t launch_attn_fwd(const AttnArgs &a, int, int cols, hipStream_t) {
    shares(a, a.H);
    need((cols == 16 || cols == 32) && a.tiles == (a.Nq + cols - 1) / cols && a.nsplit >= 1);
    need(int64_t(a.nwg) == int64_t(a.B) * a.tiles * (a.H / a.hp) * a.nsplit);
    need(a.nsplit == 1 || (a.part && a.part_ml));
    need(a.D <= 64 || cols == 16);
    return hipSuccess;
}
hipError_t launch_attn_recall(const AttnArgs &a, int dtype, int cols, hipStream_t s) {
    return launch_attn_fwd(a, dtype, cols, s);
}
hipError_t launch_attn_combine(const AttnArgs &a, int, hipStream_t) {
    need(a.nsplit > 1);
    return hipSuccess;
}
// The key pass's LDS: tables of biases (binary32) and of sums (binary64) for eight waves, buckets,
// tiles of rows, or the sums that its waves join at the end.
bool dkv_fits(const AttnArgs &a, int dtype, int cols) {
    const int dp = a.D <= 32 ? 32 : a.D <= 64 ? 64 : 128, nb2 = a.rule.nb * a.rule.nb;
    int64_t at = dtype == 1 && dp <= 64 ? int64_t(kAttnWaves) * 2 * kTile * dp * 2 : 0;
    if (a.bias)
        at += a.hp * a.head_step * ((nb2 * 4 + 15) & ~15) + cols * 16 +
              2 * (a.parts >= 2 ? 1 : 2) * a.parts * cols * 80 + ((kAttnWaves * a.head_step * nb2 * 8 + 15) & ~15);
    const int64_t end = a.parts > 1 ? int64_t(a.hp) * a.parts * cols * (dp + 4) * 4 : 0;
    return std::max(at, end) <= kLdsBytes;
}
hipError_t launch_attn_bwd(const AttnArgs &dq, const AttnArgs &dkv, int dtype, int dq_cols, int dkv_cols, hipStream_t) {
    shares(dq, dq.H);
    shares(dkv, dkv.Hkv);
    need(dq.D <= 64 || (dq_cols == 16 && dkv_cols == 16));
    need(dkv.head_step >= 1 && dkv.head_step <= dkv.group && dkv.span >= 1);
    need(int64_t(dkv.span) * dkv.spans >= dkv.tiles && dkv_fits(dkv, dtype, dkv_cols));
    need(dq.rowstat && dkv.hist);
    return hipSuccess;
}
hipError_t launch_memory_append(MemoryArgs a, int, hipStream_t) {
    need(a.count > 0);
    return hipSuccess;
}
hipError_t launch_memory_read(MemoryArgs a, int, hipStream_t) {
    need(a.count > 0);
    return hipSuccess;
}
int norm_slots(int, int C) { return C <= 256 ? 16 : C <= 1024 ? 4 : 1; }
hipError_t launch_norm_fwd(const NormArgs &a, int, hipStream_t) {
    need(a.blocks >= 1 && int64_t(a.blocks) * a.unit_rows >= a.rows);
    return hipSuccess;
}
hipError_t launch_norm_bwd(const NormArgs &a, int, hipStream_t) {
    need(a.rows == 0 || (a.blocks >= 1 && int64_t(a.gate_parts) * a.unit_rows >= a.span));
    return hipSuccess;
}

}  // namespace rex
