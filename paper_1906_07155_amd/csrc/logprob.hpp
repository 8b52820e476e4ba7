// logprob.hpp -- argument block and launchers of the class log probabilities.
#pragma once

#include "internal.hpp"

namespace rex {

// A long row's part: the largest x, and relative to it the sums of exp(x) and of x exp(x).
struct LogPart {
    float top, sum, moment;
};

struct LogprobArgs {
    const void *logits;
    const int64_t *labels;
    int64_t stride, rows;
    int32_t C, top;
    float scale;
    int32_t parts, each;            // parts of a row, classes of each
    LogPart *part;                  // [rows][parts]
    uint64_t *keys;                 // [rows][parts][top]
    float *logp, *entropy, *stats, *top_logp;
    int64_t *top_index;
    // backward
    const float *glogp, *gentropy;
    void *grad;
};

// What a workgroup holds in registers, and the classes of a part of a longer row: a chunk of 16 bytes
// fewer, since a row may begin inside one.
constexpr int kLogprobRegisters = 4096, kLogprobSpan = kLogprobRegisters - 8;
hipError_t launch_logprob_fwd(const LogprobArgs &a, int dtype, hipStream_t s);
hipError_t launch_logprob_bwd(const LogprobArgs &a, int dtype, hipStream_t s);

}  // namespace rex
