// gemm_bf16.hip -- the dense layers' products of bf16 data (gemm.hpp).
#include "gemm.hpp"

namespace rex {

template <bool TP, bool TQ>
static hipError_t run(const GemmArgs &a, const GemmPlan &p, hipStream_t s) {
    // Through registers: 4096 x 4097 x 4095 in tiles of 64 x 64 354 us, both operands transposed 446; of
    // 128 x 128 by four waves of 64 x 64 223 and 364, by eight of 64 x 32, which have half as much on its way in
    // registers, 279 and 330.
    if (!p.chunks && p.tile == kTileMiddle) {
        if constexpr (TP && TQ) return run_gemm<uint16_t, TP, TQ, 4, 2, 2, 4, false, 2>(a, s);
        else return run_gemm<uint16_t, TP, TQ, 4, 4, 2, 2, false, 2>(a, s);
    }
    if (!p.chunks) return run_gemm<uint16_t, TP, TQ, 2, 2, 2, 2, false, 2>(a, s);
    if (p.tile == kTileLarge) return run_gemm<uint16_t, TP, TQ, 8, 4, 2, 4, true, 2>(a, s);
    if (p.tile == kTileMiddle) return run_gemm<uint16_t, TP, TQ, 4, 2, 2, 4, true, 4>(a, s);
    return run_gemm<uint16_t, TP, TQ, 2, 2, 2, 2, true, 2>(a, s);
}

hipError_t launch_gemm_bf16(const GemmArgs &a, const GemmPlan &p, bool tp, bool tq, hipStream_t s) {
    if (tp && tq) return run<true, true>(a, p, s);
    if (tp) return run<true, false>(a, p, s);
    return run<false, false>(a, p, s);
}

}  // namespace rex
