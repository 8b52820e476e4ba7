// head_api.hip -- the C ABI declared in include/box_head.h.
//
// As in api.hip, every argument is checked on the host before anything is enqueued, and no
// HIP call is made on an error path.  How a product is cut up is a function of sizes, type and
// alignment alone, so the workspace functions and the calls agree on it.
#include <algorithm>
#include <cmath>

#include "box_head.h"
#include "linear.hpp"
#include "logprob.hpp"

using namespace rex;

namespace {

size_t align256(size_t x) { return (x + 255) & ~static_cast<size_t>(255); }
bool valid_dtype(int32_t d) { return d == RE_DTYPE_F32 || d == RE_DTYPE_BF16; }
int64_t dtype_size(int32_t d) { return d == RE_DTYPE_BF16 ? 2 : 4; }
bool aligned(const void *p, uintptr_t n) { return reinterpret_cast<uintptr_t>(p) % n == 0; }
re_status_t from_hip(hipError_t e) { return e == hipSuccess ? RE_OK : RE_ERR_DEVICE; }

re_status_t check_workspace(const void *ws, size_t have, size_t need) {
    if (need == 0) return RE_OK;
    if (!ws || have < need || !aligned(ws, 256)) return RE_ERR_WORKSPACE;
    return RE_OK;
}

// One operand of a product: rows x cols elements, cols adjacent.
struct Matrix {
    const void *p;
    int64_t rows, cols, stride;
};
// 16-byte chunks of rows and nothing else: what the fast kernels read.
bool chunks(const Matrix &x, int64_t size) {
    return aligned(x.p, 16) && x.cols * size % 16 == 0 && x.stride * size % 16 == 0;
}

struct Product {
    GemmArgs a;
    GemmPlan plan;
    bool tp, tq, skinny, turned;
    size_t bytes;               // of partial sums
};

// out[M][N] = q p^T, with q [M][K], or transposed [K][M], and p [N][K] or [K][N].
//
// What a cut takes is estimated from what its kind of tile took here, in us: a step of k where the CUs are
// full (8192^3 in bf16: 256 x 256 results 875 us, 128 x 128 1045, 64 x 64 1590; 4096^3 in binary32: 128 x 64
// 1020 us, 64 x 64 1040) and of a workgroup that is alone on its CU, and what precedes and follows the steps (half of
// it is hidden behind the products of other workgroups of the CU, which 256 x 256 has none of).  Tiles
// that would start another round on the GPU's 256 CUs are cut along k until they fill it, or all are; the
// parts are written and read again at some 6 TB/s, and joined by a launch more, which costs 6 (1000 x 1024 x 1024
// in binary32 31 us in two parts, 26 in one; 300 x 256 x 1024 in bf16 15 and 9).  Steps through registers count
// 1.5 times as much in bf16, 2.0 times with an operand transposed and 1.2 times in binary32 (4096 x 4097 x 4095
// took 1.4, 2.2 and 1.1 times as long as rows of whole chunks).
struct TileCost {
    int kind, bm, bn;
    double step, alone, around;
};
const TileCost kTilesBf16[] = {{kTileLarge, 256, 256, 1.71, 1.71, 12.0}, {kTileMiddle, 128, 128, 0.51, 0.85, 3.0},
                               {kTileSmall, 64, 64, 0.20, 0.45, 1.0}};
const TileCost kTilesF32[] = {{kTileMiddle, 128, 64, 0.98, 1.4, 2.0}, {kTileSmall, 64, 64, 0.51, 0.8, 1.0}};
constexpr int64_t kCus = 256;

// Few rows, or few outputs, go from memory to the products (launch_skinny): up to 16 of them, whose sums
// may be cut into parts where they are long, or up to 64 whose sums are short enough for one launch.
// One of 1024 x 12544 in bf16 15 us that way, 17 in tiles; 16 of 2048 x 1024 9 and 15; 64 of 4096 x 1024 9 and
// 15, of 1024 x 12544 22 and 17; 6 outputs of 7397 rows x 2624 13 and 17, 16 of 16000 x 1024 14 and 12.
bool few_rows(int64_t M, int64_t N, int64_t K, int64_t size) {
    const int64_t few = std::min(M, N), groups = (std::max(M, N) + 15) / 16, steps = (K + 31) / 32;
    if (few <= 16) return groups <= 2 * kCus || steps >= 64;
    return few <= kSkinnyRows && groups <= 2 * kCus && few * steps * size <= 8192;
}

void plan_product(Product &g, const Matrix &p, bool tp, const Matrix &q, bool tq, int32_t dtype, bool smooth) {
    const int64_t size = dtype_size(dtype), step = 128 / size;
    g = Product{};
    GemmArgs &a = g.a;
    a.p = p.p;
    a.q = q.p;
    a.ldp = p.stride * size;
    a.ldq = q.stride * size;
    a.N = static_cast<int32_t>(tp ? p.cols : p.rows);
    a.M = static_cast<int32_t>(tq ? q.cols : q.rows);
    a.K = static_cast<int32_t>(tp ? p.rows : p.cols);
    a.split = 1;
    g.tp = tp;
    g.tq = tq;
    g.plan.chunks = chunks(p, size) && chunks(q, size);
    const int64_t M = a.M, N = a.N, K = a.K;
    if (few_rows(M, N, K, size) && !tp && !tq && g.plan.chunks && K % 8 == 0) {
        g.skinny = true;
        g.turned = N < M;
        const int64_t groups = (std::max(M, N) + 15) / 16, steps = (K + 31) / 32;
        if (steps >= 128) a.split = static_cast<int32_t>(std::max<int64_t>(1, std::min<int64_t>(kCus / groups, steps / 32)));
        a.steps = static_cast<int32_t>((steps + a.split - 1) / a.split);
        a.split = static_cast<int32_t>((steps + a.steps - 1) / a.steps);
        g.bytes = a.split > 1 ? align256(static_cast<size_t>(a.split) * M * N * 4) : 0;
        return;
    }
    const bool bf16 = dtype == RE_DTYPE_BF16;
    const TileCost *all = bf16 ? kTilesBf16 : kTilesF32;
    const int count = bf16 ? 3 : 2;
    const int64_t steps = (K + step - 1) / step;
    const double slow = g.plan.chunks ? 1.0 : !bf16 ? 1.2 : tp || tq ? 2.0 : 1.5;
    double best = -1;
    for (int i = g.plan.chunks ? 0 : 1; i < count; ++i) {       // (through registers: the second and third, gemm_*.hip)
        const TileCost &t = all[i];
        const int64_t tm = (M + t.bm - 1) / t.bm, tn = (N + t.bn - 1) / t.bn, tiles = tm * tn;
        // us of n workgroups of k steps each
        const auto run = [&](int64_t n, int64_t k) {
            const double rounds = double((n + kCus - 1) / kCus);
            return double(k) * slow * std::max(n > 0 ? t.alone : 0.0, rounds * t.step) + rounds * t.around * (smooth ? 1.8 : 1.0);
        };
        for (int some = 0; some < 2; ++some) {       // parts of all tiles, or of those past full rounds
            const int64_t whole = some ? tiles / kCus * kCus : 0, parted = tiles - whole;
            if (some && (whole == 0 || parted == 0)) continue;
            for (int64_t split = 1; split <= 64; ++split) {
                if (split > 1 && (steps / split < 4 || parted * split > 8 * kCus)) break;
                const int64_t each = (steps + split - 1) / split;
                if ((steps + each - 1) / each != split || (some && split == 1)) continue;
                double us = run(whole, steps) + run(parted * split, each);
                if (split > 1) us += 6.0 + 8e-6 / 6.0 * double(split * parted) * t.bm * t.bn;
                if (best >= 0 && us >= best) continue;
                best = us;
                g.plan.tile = t.kind;
                g.plan.bm = t.bm;
                g.plan.bn = t.bn;
                a.tiles_m = static_cast<int32_t>(tm);
                a.tiles_n = static_cast<int32_t>(tn);
                a.whole = static_cast<int32_t>(split == 1 ? tiles : whole);
                a.parted = static_cast<int32_t>(split == 1 ? 0 : parted);
                a.split = static_cast<int32_t>(split);
                a.steps = static_cast<int32_t>(each);
            }
        }
    }
    a.grid_whole = (a.whole + 7) / 8 * 8;
    g.bytes = align256(static_cast<size_t>(a.split) * a.parted * g.plan.bm * g.plan.bn * 4);
}

re_status_t run_product(Product &g, void *out, void *ws, int32_t dtype, hipStream_t s) {
    GemmArgs &a = g.a;
    a.out = out;
    a.part = static_cast<float *>(ws);
    const int64_t size = dtype_size(dtype);
    a.vec = !g.turned && a.N % 4 == 0 && aligned(out, 4 * size) &&
            (!a.residual || (a.ldr % 4 == 0 && aligned(a.residual, 4 * size))) && aligned(a.slope, 4 * size);
    hipError_t e;
    if (g.skinny) e = launch_skinny(a, dtype, g.turned, s);
    else if (dtype == RE_DTYPE_BF16) e = launch_gemm_bf16(a, g.plan, g.tp, g.tq, s);
    else e = launch_gemm_f32(a, g.plan, g.tp, g.tq, s);
    if (e == hipSuccess && a.split > 1) e = g.skinny ? launch_skinny_join(a, dtype, s) : launch_gemm_join(a, g.plan, dtype, s);
    return from_hip(e);
}

re_status_t check_linear(const linear_act_t *d) {
    if (!d || !valid_dtype(d->dtype)) return RE_ERR_INVALID_ARG;
    if (d->act < RE_ACT_NONE || d->act > RE_ACT_SILU) return RE_ERR_INVALID_ARG;
    if (d->rows < 0 || d->ins < 1 || d->outs < 1) return RE_ERR_INVALID_ARG;
    const uintptr_t size = static_cast<uintptr_t>(dtype_size(d->dtype));
    if (d->bias && (!valid_dtype(d->bias_dtype) || (d->bias_dtype == RE_DTYPE_BF16 && d->dtype != RE_DTYPE_BF16) ||
                    !aligned(d->bias, static_cast<uintptr_t>(dtype_size(d->bias_dtype)))))
        return RE_ERR_INVALID_ARG;
    if (!d->weight || (d->rows > 0 && !d->x)) return RE_ERR_INVALID_ARG;
    for (const void *p : {d->x, d->weight, d->residual})
        if (!aligned(p, size)) return RE_ERR_INVALID_ARG;
    const int64_t most = int64_t(1) << 40;
    const int64_t xs = d->rows > 1 ? d->x_stride : 0, ws = d->outs > 1 ? d->weight_stride : 0;
    for (int64_t v : {xs, ws, d->residual && d->rows > 1 ? d->residual_stride : 0})
        if (v < 0 || v > most) return RE_ERR_INVALID_ARG;
    if (d->rows > INT32_MAX || d->ins > RE_LINEAR_MAX_SIZE || d->outs > RE_LINEAR_MAX_SIZE) return RE_ERR_UNSUPPORTED;
    for (int64_t v : {xs, ws, d->ins, d->outs})
        if (256 * v * static_cast<int64_t>(size) >= kBufMaxBytes) return RE_ERR_UNSUPPORTED;
    // a launch has fewer than 2^32 threads: 256 for every 64 x 64 results at most, and for some tiles more
    const auto tiles = [](int64_t m, int64_t n) { return double((m + 63) / 64) * double((n + 63) / 64); };
    for (double t : {tiles(d->rows, d->outs), tiles(d->rows, d->ins), tiles(d->outs, d->ins)})
        if (t > double((1 << 24) - 16)) return RE_ERR_UNSUPPORTED;
    return RE_OK;
}

// Rows of a matrix with one row, or none, have no stride.
Matrix matrix(const void *p, int64_t rows, int64_t cols, int64_t stride) {
    return Matrix{p, rows, cols, rows > 1 ? stride : cols};
}

// Runs of rows for the column sums: about 1024 workgroups, but 16 rows at least.
void plan_slope(SlopeArgs &a, int64_t size) {
    const int64_t wide = (a.N + 1024 / size - 1) / (1024 / size);      // strips of 64 chunks of 16 bytes
    const int64_t blocks = std::max<int64_t>(1, std::min<int64_t>({1024 / wide, 512, (a.M + 15) / 16}));
    a.run = static_cast<int32_t>((a.M + blocks - 1) / blocks);
    a.blocks = a.run > 0 ? static_cast<int32_t>((a.M + a.run - 1) / a.run) : 0;
}

struct Backward {
    SlopeArgs slope;
    Product x, weight;
    size_t g_bytes, part_bytes, bytes;
};
// g: the gradient of t, grad_y or in the workspace.
void plan_backward(const linear_act_t *d, const void *grad_y, Backward &b) {
    const int64_t size = dtype_size(d->dtype);
    b = Backward{};
    b.slope.M = d->rows;
    b.slope.N = static_cast<int32_t>(d->outs);
    plan_slope(b.slope, size);
    const Matrix g = matrix(grad_y, d->rows, d->outs, d->outs);
    const Matrix w = matrix(d->weight, d->outs, d->ins, d->weight_stride);
    const Matrix x = matrix(d->x, d->rows, d->ins, d->x_stride);
    if (d->rows > 0) {
        plan_product(b.x, w, true, g, false, d->dtype, false);
        plan_product(b.weight, x, true, g, true, d->dtype, false);
    }
    b.g_bytes = d->act == RE_ACT_NONE ? 0 : align256(static_cast<size_t>(d->rows) * d->outs * size);
    b.part_bytes = d->bias ? align256(static_cast<size_t>(b.slope.blocks) * d->outs * 4) : 0;
    b.bytes = b.g_bytes + b.part_bytes + std::max(b.x.bytes, b.weight.bytes);
}

re_status_t logprob_args(const class_logprob_t *d, LogprobArgs *a) {
    *a = LogprobArgs{};
    if (!d || !valid_dtype(d->dtype)) return RE_ERR_INVALID_ARG;
    if (d->rows < 0 || d->classes < 1) return RE_ERR_INVALID_ARG;
    if (d->top < 0 || d->top > RE_LOGPROB_MAX_TOP || d->top > d->classes) return RE_ERR_INVALID_ARG;
    if (!std::isfinite(d->scale) || !(d->scale > 0.0f)) return RE_ERR_INVALID_ARG;
    if (d->rows > 0 && (!d->logits || !d->labels)) return RE_ERR_INVALID_ARG;
    if (!aligned(d->logits, static_cast<uintptr_t>(dtype_size(d->dtype))) || !aligned(d->labels, 8))
        return RE_ERR_INVALID_ARG;
    if (d->rows > 1 && (d->stride < 0 || d->stride > (int64_t(1) << 40))) return RE_ERR_INVALID_ARG;
    if (d->classes > RE_LOGPROB_MAX_CLASSES) return RE_ERR_UNSUPPORTED;
    a->logits = d->logits;
    a->labels = d->labels;
    a->stride = d->rows > 1 ? d->stride : 0;
    a->rows = d->rows;
    a->C = static_cast<int32_t>(d->classes);
    a->top = d->top;
    a->scale = d->scale;
    a->parts = static_cast<int32_t>((d->classes + kLogprobSpan - 1) / kLogprobSpan);
    a->each = static_cast<int32_t>(((d->classes + a->parts - 1) / a->parts + 7) / 8 * 8);
    // a row or part may be a workgroup's work, and a launch has fewer than 2^32 threads
    if (d->rows > RE_LOGPROB_MAX_ROWS / a->parts) return RE_ERR_UNSUPPORTED;
    return RE_OK;
}
size_t logprob_part_bytes(const LogprobArgs &a) {
    return a.parts > 1 ? align256(static_cast<size_t>(a.rows) * a.parts * sizeof(LogPart)) : 0;
}
size_t logprob_bytes(const LogprobArgs &a) {
    return a.parts > 1 ? logprob_part_bytes(a) + align256(static_cast<size_t>(a.rows) * a.parts * a.top * 8) : 0;
}

}  // namespace

extern "C" {

re_status_t linear_act_workspace_size(const linear_act_t *d, int32_t backward, size_t *bytes) {
    if (!bytes) return RE_ERR_INVALID_ARG;
    const re_status_t st = check_linear(d);
    if (st != RE_OK) return st;
    if (backward) {
        // without an activation grad_y itself is an operand, whose alignment is not known yet
        Backward b, c;
        plan_backward(d, nullptr, b);
        plan_backward(d, reinterpret_cast<const void *>(uintptr_t(d->act == RE_ACT_NONE ? 4 : 0)), c);
        *bytes = std::max(b.bytes, c.bytes);
    } else {
        *bytes = 0;
        if (d->rows > 0) {
            Product g;
            plan_product(g, matrix(d->weight, d->outs, d->ins, d->weight_stride), false,
                         matrix(d->x, d->rows, d->ins, d->x_stride), false, d->dtype, d->act >= RE_ACT_GELU);
            *bytes = g.bytes;
        }
    }
    return RE_OK;
}

re_status_t linear_act_fwd(const linear_act_t *d, void *y, void *slope, void *workspace,
                           size_t workspace_bytes, void *stream) {
    re_status_t st = check_linear(d);
    if (st != RE_OK) return st;
    if (slope && d->act == RE_ACT_NONE) return RE_ERR_INVALID_ARG;
    const uintptr_t size = static_cast<uintptr_t>(dtype_size(d->dtype));
    if (!aligned(y, size) || !aligned(slope, d->dtype == RE_DTYPE_BF16 ? 16 : 4)) return RE_ERR_INVALID_ARG;
    if (d->rows == 0) return RE_OK;
    if (!y) return RE_ERR_INVALID_ARG;
    Product g;
    plan_product(g, matrix(d->weight, d->outs, d->ins, d->weight_stride), false,
                 matrix(d->x, d->rows, d->ins, d->x_stride), false, d->dtype, d->act >= RE_ACT_GELU);
    if ((st = check_workspace(workspace, workspace_bytes, g.bytes)) != RE_OK) return st;
    g.a.bias = d->bias;
    g.a.bias_bf16 = d->bias_dtype == RE_DTYPE_BF16;
    g.a.residual = d->residual;
    g.a.ldr = d->rows > 1 ? d->residual_stride : 0;
    g.a.slope = slope;
    g.a.act = d->act;
    return run_product(g, y, workspace, d->dtype, static_cast<hipStream_t>(stream));
}

re_status_t linear_act_bwd(const linear_act_t *d, const void *grad_y, const void *slope, const void *y,
                           void *grad_x, void *grad_weight, void *grad_bias, void *workspace,
                           size_t workspace_bytes, void *stream) {
    re_status_t st = check_linear(d);
    if (st != RE_OK) return st;
    const int64_t size = dtype_size(d->dtype);
    if (!aligned(slope, d->dtype == RE_DTYPE_BF16 ? 16 : 4)) return RE_ERR_INVALID_ARG;
    for (const void *p : {grad_y, y, static_cast<const void *>(grad_x), static_cast<const void *>(grad_weight)})
        if (!aligned(p, static_cast<uintptr_t>(size))) return RE_ERR_INVALID_ARG;
    if (grad_bias && (!d->bias || !aligned(grad_bias, static_cast<uintptr_t>(dtype_size(d->bias_dtype)))))
        return RE_ERR_INVALID_ARG;
    if (d->act == RE_ACT_NONE ? (slope || y) : (slope && y)) return RE_ERR_INVALID_ARG;
    if (y && d->act != RE_ACT_RELU) return RE_ERR_INVALID_ARG;
    if (d->rows > 0 && (!grad_y || (d->act != RE_ACT_NONE && !slope && !y))) return RE_ERR_INVALID_ARG;
    Backward b;
    plan_backward(d, d->act == RE_ACT_NONE ? grad_y : nullptr, b);
    if ((st = check_workspace(workspace, workspace_bytes, b.bytes)) != RE_OK) return st;
    char *ws = static_cast<char *>(workspace);
    const hipStream_t s = static_cast<hipStream_t>(stream);

    const void *g = grad_y;
    SlopeArgs &sl = b.slope;
    const bool times = d->act != RE_ACT_NONE && (grad_x || grad_weight);
    sl.gy = grad_y;
    sl.saved = d->act == RE_ACT_NONE ? nullptr : slope ? slope : y;
    sl.relu = y != nullptr;
    if (d->act != RE_ACT_NONE) g = sl.g = ws;
    sl.part = grad_bias ? reinterpret_cast<float *>(ws + b.g_bytes) : nullptr;
    sl.gbias = grad_bias;
    sl.bias_bf16 = d->bias_dtype == RE_DTYPE_BF16;
    sl.vec = d->outs * size % 16 == 0 && aligned(grad_y, 16) && aligned(sl.saved, 16);
    if ((times && d->rows > 0) || grad_bias)
        if ((st = from_hip(launch_slope(sl, d->dtype, s))) != RE_OK) return st;
    void *part = ws + b.g_bytes + b.part_bytes;
    if (grad_x && d->rows > 0) {
        b.x.a.q = g;
        if ((st = run_product(b.x, grad_x, part, d->dtype, s)) != RE_OK) return st;
    }
    if (grad_weight) {
        if (d->rows == 0) return from_hip(launch_clear(grad_weight, d->outs * d->ins * size, s));
        b.weight.a.q = g;
        if ((st = run_product(b.weight, grad_weight, part, d->dtype, s)) != RE_OK) return st;
    }
    return RE_OK;
}

re_status_t class_logprob_workspace_size(const class_logprob_t *d, size_t *bytes) {
    if (!bytes) return RE_ERR_INVALID_ARG;
    LogprobArgs a;
    const re_status_t st = logprob_args(d, &a);
    if (st != RE_OK) return st;
    *bytes = logprob_bytes(a);
    return RE_OK;
}

re_status_t class_logprob_fwd(const class_logprob_t *d, float *logp, float *entropy, float *stats,
                              float *top_logp, int64_t *top_index, void *workspace,
                              size_t workspace_bytes, void *stream) {
    LogprobArgs a;
    re_status_t st = logprob_args(d, &a);
    if (st != RE_OK) return st;
    if (!aligned(logp, 4) || !aligned(entropy, 4) || !aligned(stats, 8)) return RE_ERR_INVALID_ARG;
    if (a.rows > 0 && (!logp || !entropy || !stats)) return RE_ERR_INVALID_ARG;
    if (a.top > 0 && (!aligned(top_logp, 4) || !aligned(top_index, 8) || (a.rows > 0 && (!top_logp || !top_index))))
        return RE_ERR_INVALID_ARG;
    if (a.rows == 0) return RE_OK;
    if ((st = check_workspace(workspace, workspace_bytes, logprob_bytes(a))) != RE_OK) return st;
    a.logp = logp;
    a.entropy = entropy;
    a.stats = stats;
    a.top_logp = top_logp;
    a.top_index = top_index;
    a.part = static_cast<LogPart *>(workspace);
    a.keys = reinterpret_cast<uint64_t *>(static_cast<char *>(workspace) + logprob_part_bytes(a));
    return from_hip(launch_logprob_fwd(a, d->dtype, static_cast<hipStream_t>(stream)));
}

re_status_t class_logprob_bwd(const class_logprob_t *d, const float *grad_logp, const float *grad_entropy,
                              const float *stats, const float *entropy, void *grad_logits, void *stream) {
    LogprobArgs a;
    const re_status_t st = logprob_args(d, &a);
    if (st != RE_OK) return st;
    if (!aligned(grad_logp, 4) || !aligned(grad_entropy, 4) || !aligned(stats, 8) || !aligned(entropy, 4))
        return RE_ERR_INVALID_ARG;
    if (!aligned(grad_logits, static_cast<uintptr_t>(dtype_size(d->dtype)))) return RE_ERR_INVALID_ARG;
    if (a.rows == 0) return RE_OK;
    if (!stats || !entropy || !grad_logits) return RE_ERR_INVALID_ARG;
    a.glogp = grad_logp;
    a.gentropy = grad_entropy;
    a.stats = const_cast<float *>(stats);
    a.entropy = const_cast<float *>(entropy);
    a.grad = grad_logits;
    return from_hip(launch_logprob_bwd(a, d->dtype, static_cast<hipStream_t>(stream)));
}

}  // extern "C"
