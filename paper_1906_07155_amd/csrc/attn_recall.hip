// attn_recall.hip -- box_memory_attn_fwd's kernels.
#include "attn_fwd.hpp"

namespace rex {

hipError_t launch_attn_recall(const AttnArgs &a, int dtype, int cols, hipStream_t s) {
    if (dtype == kF32) return run_fwd_sized<float, true, 1>(a, cols, s);
    return a.terms > 1 ? run_fwd_sized<uint16_t, true, 2>(a, cols, s)
                       : run_fwd_sized<uint16_t, true, 1>(a, cols, s);
}

}  // namespace rex
