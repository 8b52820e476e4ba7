// gemm_f32.hip -- the dense layers' products of binary32 data (gemm.hpp).
#include "gemm.hpp"

namespace rex {

template <bool TP, bool TQ>
static hipError_t run(const GemmArgs &a, const GemmPlan &p, hipStream_t s) {
    // (through registers; tiles of 128 x 64 took a tenth longer)
    if (!p.chunks) return run_gemm<float, TP, TQ, 2, 2, 2, 2, false, 2>(a, s);
    if (p.tile == kTileMiddle) return run_gemm<float, TP, TQ, 4, 2, 2, 2, true, 3>(a, s);
    return run_gemm<float, TP, TQ, 2, 2, 2, 2, true, 2>(a, s);
}

hipError_t launch_gemm_f32(const GemmArgs &a, const GemmPlan &p, bool tp, bool tq, hipStream_t s) {
    if (tp && tq) return run<true, true>(a, p, s);
    if (tp) return run<true, false>(a, p, s);
    return run<false, false>(a, p, s);
}

}  // namespace rex
