// attn_dense.hip -- box_attn_fwd's kernels, and the joining of split keys.
#include "attn_fwd.hpp"

namespace rex {

namespace {

// Joins the partial results of the key splits: a thread for eight channels of one row.
// Reads nsplit * (D + 4) floats per row once: bytes bound.
template <typename T>
__global__ __launch_bounds__(256) void attn_combine_kernel(AttnArgs a) {
    using N = Num<T>;
    const int chunks = a.D / 8;
    const int64_t e = static_cast<int64_t>(blockIdx.x) * 256 + threadIdx.x;
    const int64_t rows = static_cast<int64_t>(a.B) * a.H * a.Nq;
    if (e >= rows * chunks) return;
    const int64_t r = e / chunks;
    const int ch = static_cast<int>(e - r * chunks) * 8;
    const int row = static_cast<int>(r % a.Nq), h = static_cast<int>(r / a.Nq % a.H);
    const int b = static_cast<int>(r / (static_cast<int64_t>(a.Nq) * a.H));
    const int qlen = a.qlen ? min(max(a.qlen[b], 0), a.Nq) : a.Nq;
    float sum = 0.0f, x[8] = {};
    SumRef to = load_ref(a.part_ml + r);
    if (row < qlen) {
        for (int s = 1; s < a.nsplit; ++s) reach(to, load_ref(a.part_ml + s * rows + r));
        for (int s = 0; s < a.nsplit; ++s) {
            const SumRef p = load_ref(a.part_ml + s * rows + r);
            const float f = __builtin_amdgcn_exp2f(ref_gap(p, to));
            const f32x8 y = Num<float>::load(reinterpret_cast<const char *>(
                a.part + (s * rows + r) * a.D + ch));
            sum = fmaf(p.sum, f, sum);
#pragma unroll
            for (int i = 0; i < 8; ++i) x[i] = fmaf(y[i], f, x[i]);
        }
    }
    const float inv = sum == 0.0f ? 0.0f : 1.0f / sum;
#pragma unroll
    for (int i = 0; i < 8; ++i) x[i] *= inv;
    const int64_t at = (((static_cast<int64_t>(b) * a.Nq + row) * a.H + h) * a.D + ch) * N::kSize;
    N::store(static_cast<char *>(a.out) + at, x);
    if (a.out_f32) Num<float>::store(reinterpret_cast<char *>(a.out_f32) + at * (4 / N::kSize), x);
    if (ch == 0 && a.lse)
        as_global_mut<float>(a.lse)[r] = row_lse(SumRef{to.offset, sum, to.rest});
}

}  // namespace

hipError_t launch_attn_fwd(const AttnArgs &a, int dtype, int cols, hipStream_t s) {
    if (dtype == kF32) return run_fwd_sized<float, false, 2>(a, cols, s);
    return a.terms > 2 ? run_fwd_sized<uint16_t, false, 3>(a, cols, s)
                       : run_fwd_sized<uint16_t, false, 2>(a, cols, s);
}

hipError_t launch_attn_combine(const AttnArgs &a, int dtype, hipStream_t s) {
    const int64_t n = static_cast<int64_t>(a.B) * a.H * a.Nq * (a.D / 8);
    const dim3 grid(static_cast<uint32_t>((n + 255) / 256));
    if (dtype == kBF16) hipLaunchKernelGGL((attn_combine_kernel<uint16_t>), grid, dim3(256), 0, s, a);
    else hipLaunchKernelGGL((attn_combine_kernel<float>), grid, dim3(256), 0, s, a);
    return hipGetLastError();
}

}  // namespace rex
