// linear.hpp -- argument blocks and launchers of the dense layers' kernels.
#pragma once

#include "relation.hpp"

namespace rex {

enum : int { kActNone = 0, kActRelu = 1, kActGelu = 2, kActSilu = 3 };

// One product: out[m][n] = sum_k Q(m, k) P(n, k), both operands with k adjacent in memory
// ([row][k]) or, transposed, with their rows adjacent ([k][row]).
struct GemmArgs {
    const void *p, *q;
    int64_t ldp, ldq;               // bytes from row to row, or from k to k
    void *out;                      // [M][N] dense
    int32_t M, N, K;
    int32_t tiles_m, tiles_n;       // tiles, of which the first `whole` are made by one workgroup each
    int32_t whole, grid_whole;      // (rounded up to a multiple of 8 for them)
    int32_t parted;                 // the others in `split` parts of k, of `steps` steps each
    int32_t split, steps;
    float *part;                    // [split][parted][rows and columns of a tile]; few rows: [split][M][N]
    // epilogue
    const void *bias;               // [N] or null
    const void *residual;           // [M][N], ldr elements from row to row, or null
    int64_t ldr;
    void *slope;                    // [M][N] dense or null
    int32_t bias_bf16, act;
    int32_t vec;                    // four adjacent results can be written (and residuals read) at once
};

// How a product is cut up.
enum : int { kTileLarge = 0, kTileMiddle = 1, kTileSmall = 2 };
struct GemmPlan {
    int tile, bm, bn;               // a workgroup's rows and columns
    bool chunks;                    // operands can be read 16 bytes at a time
};

hipError_t launch_gemm_bf16(const GemmArgs &a, const GemmPlan &p, bool tp, bool tq, hipStream_t s);
hipError_t launch_gemm_f32(const GemmArgs &a, const GemmPlan &p, bool tp, bool tq, hipStream_t s);
hipError_t launch_gemm_join(const GemmArgs &a, const GemmPlan &p, int dtype, hipStream_t s);
hipError_t launch_skinny_join(const GemmArgs &a, int dtype, hipStream_t s);
// A few rows against [N][K], or few outputs of many rows (turned): what there is much of goes from
// memory straight to the products.
constexpr int kSkinnyRows = 64;
hipError_t launch_skinny(const GemmArgs &a, int dtype, bool turned, hipStream_t s);

struct SlopeArgs {
    const void *gy, *saved;         // [M][N] dense; saved null: slope 1
    void *g;                        // gy * slope, or null
    float *part;                    // [blocks][N]: column sums of runs of rows, or null
    void *gbias;                    // [N]
    int32_t bias_bf16;
    int32_t relu;                   // `saved` is the layer's result, not the slope
    int32_t N;
    int64_t M;
    int32_t blocks, run;            // runs of `run` rows
    int32_t vec;
};
hipError_t launch_slope(const SlopeArgs &a, int dtype, hipStream_t s);
hipError_t launch_clear(void *p, int64_t bytes, hipStream_t s);      // an even number of them

}  // namespace rex
