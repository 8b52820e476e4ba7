// linear.hip -- the dense layers' kernels beside the tiled products: few rows, the joining of
// parts, the upstream gradient times the activation's slope.
#include "epilogue.hpp"

namespace rex {

// ---------------------------------------------------------------------------
// Few rows
// ---------------------------------------------------------------------------
// The weights are read once, by all of the GPU, and that is what bounds it: a workgroup takes 16
// outputs, its waves every 16th step of 32 inputs, straight from memory into the products' operands.
// The rows are the products' columns, so one to 64 of them cost the same weights.  Few outputs of many
// rows are the same the other way round (TURNED): rows come from memory, weights are the columns.
// A row of 1024 x 1024 in bf16 takes 4.6 us: a launch, two dependent loads and the meeting of 16 waves.
constexpr int kSkinnyWaves = 16;

template <typename T, int NQ, bool TURNED>
__global__ __launch_bounds__(kSkinnyWaves * 64) void skinny_kernel(GemmArgs a) {
    using N = Num<T>;
    using Frag = typename N::Frag;
    __shared__ f32x4 sums[kSkinnyWaves][NQ][64];
    const int lane = threadIdx.x & 63, n = lane & 15, g = lane >> 4;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int n0 = blockIdx.x * 16, part = blockIdx.y;
    // the many rows and the few
    const int many = TURNED ? a.M : a.N, few = TURNED ? a.N : a.M;
    const int64_t ldp = TURNED ? a.ldq : a.ldp, ldq = TURNED ? a.ldp : a.ldq;
    const auto pr = make_rsrc(static_cast<const char *>(TURNED ? a.q : a.p) + n0 * ldp, kBufMaxBytes - 1);
    const auto qr = make_rsrc(TURNED ? a.p : a.q, kBufMaxBytes - 1);
    const uint32_t poff = n0 + n < many ? static_cast<uint32_t>(n * ldp) : kBufOOB;
    uint32_t qoff[NQ];
#pragma unroll
    for (int t = 0; t < NQ; ++t) qoff[t] = 16 * t + n < few ? static_cast<uint32_t>((16 * t + n) * ldq) : kBufOOB;

    f32x4 acc[NQ] = {};
    const int all = (a.K + 31) / 32, first = part * a.steps, end = min(first + a.steps, all);
    constexpr int kAhead = NQ == 1 ? 4 : 2;
    for (int step = first + wave; step < end; step += kAhead * kSkinnyWaves) {
        Frag p[kAhead], q[kAhead][NQ];
#pragma unroll
        for (int u = 0; u < kAhead; ++u) {
            const int k = (step + u * kSkinnyWaves) * 32 + 8 * g;
            const bool in = step + u * kSkinnyWaves < end && k < a.K;
            // (offsets of a row are below the range, and two marks do not wrap)
            const uint32_t at = in ? k * N::kSize : kBufOOB;
            p[u] = N::load(pr, poff + at, 0);
#pragma unroll
            for (int t = 0; t < NQ; ++t) q[u][t] = N::load(qr, qoff[t] + at, 0);
        }
#pragma unroll
        for (int u = 0; u < kAhead; ++u)
#pragma unroll
            for (int t = 0; t < NQ; ++t) acc[t] = N::mma(p[u], q[u][t], acc[t]);
    }
    asm volatile("s_nop 15" ::: "memory");   // (between products and a use behind a branch)
#pragma unroll
    for (int t = 0; t < NQ; ++t) sums[wave][t][lane] = acc[t];
    __syncthreads();
    if (wave >= NQ) return;
    f32x4 x = sums[0][wave][lane];
#pragma unroll
    for (int w = 1; w < kSkinnyWaves; ++w) x += sums[w][wave][lane];
    if constexpr (TURNED) {             // four rows of one output
        const int col = 16 * wave + n;
        if (col >= a.N) return;
        const float bias = a.bias && a.split == 1 ? load_bias(a, col)[0] : 0.0f;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const int m = n0 + 4 * g + i;
            if (m >= a.M) return;
            const int64_t at = static_cast<int64_t>(m) * a.N + col;
            if (a.split > 1) as_global_mut<float>(a.part)[static_cast<int64_t>(part) * a.M * a.N + at] = x[i];
            else finish4<T>(a, 1, at, m * a.ldr + col, f32x4{x[i] + bias, 0.0f, 0.0f, 0.0f});
        }
        return;
    }
    const int m = 16 * wave + n, to = n0 + 4 * g;
    if (m >= a.M || to >= a.N) return;
    const int64_t at = static_cast<int64_t>(m) * a.N + to;
    if (a.split > 1) {
        float *sums = a.part + static_cast<int64_t>(part) * a.M * a.N + at;
#pragma unroll
        for (int i = 0; i < 4; ++i)
            if (to + i < a.N) as_global_mut<float>(sums)[i] = x[i];
    } else finish4<T>(a, a.N - to, at, m * a.ldr + to, x + load_bias(a, to));
}

template <typename T, bool TURNED>
static void run_skinny(const GemmArgs &a, hipStream_t s) {
    const int few = TURNED ? a.N : a.M;
    const dim3 grid(((TURNED ? a.M : a.N) + 15) / 16, a.split);
    if (few <= 16) skinny_kernel<T, 1, TURNED><<<grid, kSkinnyWaves * 64, 0, s>>>(a);
    else if (few <= 32) skinny_kernel<T, 2, TURNED><<<grid, kSkinnyWaves * 64, 0, s>>>(a);
    else skinny_kernel<T, 4, TURNED><<<grid, kSkinnyWaves * 64, 0, s>>>(a);
}

hipError_t launch_skinny(const GemmArgs &a, int dtype, bool turned, hipStream_t s) {
    if (dtype == kBF16) turned ? run_skinny<uint16_t, true>(a, s) : run_skinny<uint16_t, false>(a, s);
    else turned ? run_skinny<float, true>(a, s) : run_skinny<float, false>(a, s);
    return hipGetLastError();
}

// ---------------------------------------------------------------------------
// Parts of k
// ---------------------------------------------------------------------------

// A thread for four adjacent results of a tile that was made in parts, which it adds in order.  1000 x 1024
// in eight parts 8 us (4.2 TB/s), two of them a launch.  (The last workgroup of a tile adding up its
// parts would spare the launch, for a fence and a count in memory that the caller has to clear.)
template <typename T>
__global__ __launch_bounds__(256) void join_kernel(GemmArgs a, int bm, int bn) {
    const int quads = bm * bn / 4, tile = blockIdx.x / (quads / 256), at = blockIdx.x % (quads / 256) * 256 + threadIdx.x;
    int id = a.whole + tile;
    const int band = id / (8 * a.tiles_n), rows_of = min(8, a.tiles_m - 8 * band);
    id -= band * 8 * a.tiles_n;
    const int m = (8 * band + id % rows_of) * bm + at / (bn / 4), n = id / rows_of * bn + at % (bn / 4) * 4;
    if (m >= a.M || n >= a.N) return;
    const f32x4 *from = reinterpret_cast<const f32x4 *>(a.part) + static_cast<int64_t>(tile) * quads + at;
    f32x4 x = {};
#pragma unroll 8
    for (int i = 0; i < a.split; ++i) x += as_global<f32x4>(from)[static_cast<int64_t>(i) * a.parted * quads];
    finish4<T>(a, a.N - n, static_cast<int64_t>(m) * a.N + n, m * a.ldr + n, x + load_bias(a, n));
}

hipError_t launch_gemm_join(const GemmArgs &a, const GemmPlan &p, int dtype, hipStream_t s) {
    const uint32_t grid = static_cast<uint32_t>(a.parted) * (p.bm * p.bn / 1024);
    if (dtype == kBF16) join_kernel<uint16_t><<<grid, 256, 0, s>>>(a, p.bm, p.bn);
    else join_kernel<float><<<grid, 256, 0, s>>>(a, p.bm, p.bn);
    return hipGetLastError();
}

template <typename T>
__global__ __launch_bounds__(256) void skinny_join_kernel(GemmArgs a) {
    const int quads = (a.N + 3) / 4, at = blockIdx.x * 256 + threadIdx.x, m = at / quads, n = at % quads * 4;
    if (m >= a.M) return;
    const int64_t size = static_cast<int64_t>(a.M) * a.N, to = static_cast<int64_t>(m) * a.N + n;
    f32x4 x = {};
    for (int i = 0; i < a.split; ++i)
#pragma unroll
        for (int e = 0; e < 4; ++e)
            if (n + e < a.N) x[e] += as_global<float>(a.part)[i * size + to + e];
    finish4<T>(a, a.N - n, to, m * a.ldr + n, x + load_bias(a, n));
}

hipError_t launch_skinny_join(const GemmArgs &a, int dtype, hipStream_t s) {
    const uint32_t grid = (static_cast<uint32_t>(a.M) * ((a.N + 3) / 4) + 255) / 256;
    if (dtype == kBF16) skinny_join_kernel<uint16_t><<<grid, 256, 0, s>>>(a);
    else skinny_join_kernel<float><<<grid, 256, 0, s>>>(a);
    return hipGetLastError();
}

// ---------------------------------------------------------------------------
// Upstream gradient times slope, and its column sums
// ---------------------------------------------------------------------------
// One pass over both, a lane 16 bytes of a row at a time; the sums over a run of rows are taken
// before the product is rounded.  `lanes` (a power of two) lanes take a row, so that narrow layers
// use whole waves too.  Bytes bound it: 16000 x 2048 in bf16 with slopes of 24 bits 38 us, 229 MB at 6 TB/s.
//
// g is rounded to bf16, where the data is, for the two products that follow: with an activation other than
// max(t, 0) their results are then off by two roundings of 2^-9 in the mean, 2.3e-3 of their norm instead
// of 1.7e-3 (torch's own bf16 layers, whose activation's gradient is a bf16 tensor: 2.4e-3, and so are their y and
// bias gradients, which are 1.7e-3 here).  In two parts it would be one, for twice the products (70 and 81 us
// more at that size).

// 16 bytes of them
template <typename T, int V> __device__ __forceinline__ void load_run(const T *p, float *x) {
    using Chunk = T __attribute__((ext_vector_type(V)));
    const Chunk c = *(const REX_GLOBAL Chunk *)(p);
#pragma unroll
    for (int i = 0; i < V; ++i) {
        if constexpr (sizeof(T) == 2) x[i] = bf16_to_f32(c[i]);
        else x[i] = c[i];
    }
}

template <typename T, int V, bool SLOPE, bool RELU>
__global__ __launch_bounds__(256) void slope_kernel(SlopeArgs a, int lanes, int strips) {
    __shared__ float sums[256 * V];
    const int strip = blockIdx.x % strips, block = blockIdx.x / strips;
    const int slot = threadIdx.x / lanes, slots = 256 / lanes;
    const int n = (strip * lanes + threadIdx.x % lanes) * V;
    const int64_t first = static_cast<int64_t>(block) * a.run, end = min(first + a.run, a.M);
    float sum[V] = {};
    if (n < a.N) {
#pragma unroll 4
        for (int64_t m = first + slot; m < end; m += slots) {
            const int64_t at = m * a.N + n;
            float g[V], f[V];
            if constexpr (V == 1) {
                g[0] = load_f32<T>(as_global<T>(a.gy) + at);
                if (SLOPE && RELU) f[0] = load_f32<T>(as_global<T>(a.saved) + at);
            } else {
                load_run<T, V>(static_cast<const T *>(a.gy) + at, g);
                if (SLOPE && RELU) load_run<T, V>(static_cast<const T *>(a.saved) + at, f);
            }
            if (SLOPE && !RELU) Slope<T>::template load<V>(a.saved, a.M * a.N, at, f);
            if (SLOPE) {
#pragma unroll
                for (int i = 0; i < V; ++i) g[i] = RELU ? (f[i] <= 0.0f ? 0.0f : g[i]) : g[i] * f[i];
                if constexpr (V == 1) {
                    store_f32<T>(as_global_mut<T>(a.g) + at, g[0]);
                } else if constexpr (sizeof(T) == 2) {
                    Num<T>::store(reinterpret_cast<char *>(static_cast<T *>(a.g) + at), g);
                } else {
                    Num<T>::store4(reinterpret_cast<char *>(static_cast<T *>(a.g) + at), f32x4{g[0], g[1], g[2], g[3]});
                }
            }
#pragma unroll
            for (int i = 0; i < V; ++i) sum[i] += g[i];
        }
    }
    if (!a.part) return;
#pragma unroll
    for (int i = 0; i < V; ++i) sums[threadIdx.x * V + i] = sum[i];
    __syncthreads();
    // column c of the strip: its slots in order
    for (int c = threadIdx.x; c < lanes * V; c += 256) {
        float x = 0.0f;
        for (int s = 0; s < slots; ++s) x += sums[s * lanes * V + c];
        const int to = strip * lanes * V + c;
        if (to < a.N) as_global_mut<float>(a.part)[static_cast<int64_t>(block) * a.N + to] = x;
    }
}

// 16 columns of a workgroup, 16 threads to each.
__global__ __launch_bounds__(256) void columns_kernel(SlopeArgs a) {
    __shared__ float sums[256];
    const int c = threadIdx.x & 15, t = threadIdx.x >> 4, n = blockIdx.x * 16 + c;
    float x = 0.0f;
    if (n < a.N) {
#pragma unroll 4
        for (int b = t; b < a.blocks; b += 16) x += as_global<float>(a.part)[static_cast<int64_t>(b) * a.N + n];
    }
    sums[threadIdx.x] = x;
    __syncthreads();
    if (threadIdx.x >= 16 || n >= a.N) return;
#pragma unroll
    for (int i = 1; i < 16; ++i) x += sums[i * 16 + c];
    if (a.bias_bf16) as_global_mut<uint16_t>(a.gbias)[n] = f32_to_bf16(x);
    else as_global_mut<float>(a.gbias)[n] = x;
}

template <typename T, int V>
static void run_slope(const SlopeArgs &a, hipStream_t s) {
    int lanes = 1;
    while (lanes < 64 && lanes * V < a.N) lanes *= 2;
    const int strips = (a.N + lanes * V - 1) / (lanes * V);
    const uint32_t grid = static_cast<uint32_t>(strips) * a.blocks;
    if (!a.saved) slope_kernel<T, V, false, false><<<grid, 256, 0, s>>>(a, lanes, strips);
    else if (a.relu) slope_kernel<T, V, true, true><<<grid, 256, 0, s>>>(a, lanes, strips);
    else slope_kernel<T, V, true, false><<<grid, 256, 0, s>>>(a, lanes, strips);
}

hipError_t launch_slope(const SlopeArgs &a, int dtype, hipStream_t s) {
    if (a.blocks > 0) {
        if (dtype == kBF16 && a.vec) run_slope<uint16_t, 8>(a, s);
        else if (dtype == kBF16) run_slope<uint16_t, 1>(a, s);
        else if (a.vec) run_slope<float, 4>(a, s);
        else run_slope<float, 1>(a, s);
        const hipError_t e = hipGetLastError();
        if (e != hipSuccess) return e;
    }
    if (a.gbias) columns_kernel<<<(a.N + 15) / 16, 256, 0, s>>>(a);
    return hipGetLastError();
}

__global__ __launch_bounds__(256) void clear_kernel(uint16_t *p, int64_t n) {
    for (int64_t i = blockIdx.x * int64_t(256) + threadIdx.x; i < n; i += int64_t(gridDim.x) * 256)
        as_global_mut<uint16_t>(p)[i] = 0;
}

hipError_t launch_clear(void *p, int64_t bytes, hipStream_t s) {
    const int64_t n = bytes / 2, grid = (n + 255) / 256;
    clear_kernel<<<static_cast<uint32_t>(grid < 4096 ? grid : 4096), 256, 0, s>>>(static_cast<uint16_t *>(p), n);
    return hipGetLastError();
}

}  // namespace rex
