// attn_recall.hip -- box_memory_attn_fwd's kernels.
#include "attn_fwd.hpp"

namespace rex {

hipError_t launch_attn_recall(const AttnArgs &a, int dtype, int cols, hipStream_t s) {
    return dtype == kF32 ? run_fwd_sized<float, true, 2>(a, cols, s) : run_fwd_sized<uint16_t, true, 2>(a, cols, s);
}

}  // namespace rex
