// norm.hip -- the norms around a block with its gate and residual sum (gated_norm_fwd,
// gated_norm_bwd):  y = x + alpha * gate * N1(branch),  u = N2(y).
//
// A row stays in the registers of TPR threads, V chunks of 16 bytes each, from its one read
// to its one write: mean and variance are two sums over what is already there (the variance
// of the deviations, not of the squares).  Both directions are bound by the bytes of
// the rows.  The column sums of the backward are kept in registers over all the rows of a
// workgroup and added up in a fixed order by a second kernel.
//
// Measured, 16000 rows of 1024 channels, bf16: forward 27 us (131 MB, 4.9 TB/s, the rate of a
// large copy), backward 54 us (197 MB, 3.6 TB/s: its column sums, which it keeps for biases and gates
// where the call has none too, leave 16 waves on a CU) and 4 us for the sums.  The same in binary32:
// 67 us (262 MB, 3.9 TB/s), 95 (393 MB, 4.1 TB/s) and 5.  1000 rows of 256: 4 us, a launch.
#include "attn.hpp"

namespace rex {

namespace {

// A workgroup: several rows side by side, or one row of up to 1024 threads.
constexpr int threads_of(int tpr) { return tpr > 256 ? tpr : 256; }

template <typename T> struct Chunk;    // the elements of 16 bytes
template <> struct Chunk<uint16_t> { static constexpr int kN = 8; };
template <> struct Chunk<float> { static constexpr int kN = 4; };

template <typename T, int E>
__device__ __forceinline__ void store_row(void *row, int col, int C, bool vec, const float *x) {
    if (vec) {
        if (col >= C) return;
        if constexpr (E == 8) {
            bf16x8 f;
#pragma unroll
            for (int i = 0; i < 8; ++i) f[i] = static_cast<__bf16>(x[i]);
            *(REX_GLOBAL bf16x8 *)(static_cast<char *>(row) + col * 2) = f;
        } else {
            *(REX_GLOBAL f32x4 *)(static_cast<char *>(row) + col * 4) = f32x4{x[0], x[1], x[2], x[3]};
        }
    } else {
#pragma unroll
        for (int i = 0; i < E; ++i)
            if (col + i < C) store_f32<T>(as_global_mut<T>(row) + col + i, x[i]);
    }
}

// E parameters (binary32) or `none` where there is no such array; vec: 16 bytes at a time.
template <int E>
__device__ __forceinline__ void load_param(const float *p, int col, int C, bool vec, float none, float *x) {
#pragma unroll
    for (int i = 0; i < E; ++i) x[i] = none;
    if (!p) return;
    if (vec) {
        if (col < C) {
#pragma unroll
            for (int i = 0; i < E; i += 4) {
                const f32x4 f = *(const REX_GLOBAL f32x4 *)(p + col + i);
                x[i] = f[0], x[i + 1] = f[1], x[i + 2] = f[2], x[i + 3] = f[3];
            }
        }
    } else {
#pragma unroll
        for (int i = 0; i < E; ++i)
            if (col + i < C) x[i] = as_global<float>(p)[col + i];
    }
}

// Sums of two values over the TPR threads of a row; every one of them gets both.
template <int TPR>
__device__ __forceinline__ void row_sum(float &a, float &b, f32x2 (&mem)[2][16], int &turn) {
#pragma unroll
    for (int d = 1; d < (TPR < 64 ? TPR : 64); d <<= 1) {
        a += __shfl_xor(a, d);
        b += __shfl_xor(b, d);
    }
    if constexpr (TPR > 64) {
        constexpr int kWaves = TPR / 64;
        const int wave = threadIdx.x >> 6, first = wave / kWaves * kWaves;
        if ((threadIdx.x & 63) == 0) mem[turn][wave] = f32x2{a, b};
        __syncthreads();
        a = b = 0.0f;
#pragma unroll
        for (int w = 0; w < kWaves; ++w) {
            a += mem[turn][first + w][0];
            b += mem[turn][first + w][1];
        }
        turn ^= 1;        // the next sum writes elsewhere, so one barrier is enough
    }
}

// What a thread has of a row as it was read: conversion waits until it is used.
template <typename T, int V>
struct RowChunk {
    u32x4 v[V];
};
template <typename T, int TPR, int V>
__device__ __forceinline__ RowChunk<T, V> fetch(const void *base, int64_t row, int64_t stride, int t, int C,
                                                bool vec) {
    constexpr int E = Chunk<T>::kN;
    const char *p = static_cast<const char *>(base) + row * stride * static_cast<int>(sizeof(T));
    RowChunk<T, V> r;
#pragma unroll
    for (int k = 0; k < V; ++k) {
        const int col = (k * TPR + t) * E;
        r.v[k] = u32x4{};
        if (vec) {
            if (col < C) r.v[k] = *(const REX_GLOBAL u32x4 *)(p + col * static_cast<int>(sizeof(T)));
        } else {
#pragma unroll
            for (int i = 0; i < E; ++i)
                if (col + i < C) {
                    const uint32_t bits = as_global<T>(p)[col + i];
                    if constexpr (E == 8) r.v[k][i >> 1] |= bits << (16 * (i & 1));
                }
            if constexpr (E == 4) {
#pragma unroll
                for (int i = 0; i < E; ++i)
                    if (col + i < C) r.v[k][i] = as_global<uint32_t>(p)[col + i];
            }
        }
    }
    return r;
}
template <typename T, int V>
__device__ __forceinline__ float value(const RowChunk<T, V> &r, int k, int i) {
    if constexpr (sizeof(T) == 2) return __uint_as_float(i & 1 ? r.v[k][i >> 1] & 0xffff0000u : r.v[k][i >> 1] << 16);
    else return __uint_as_float(r.v[k][i]);
}

// Rows go to the workgroups in runs; a thread keeps its columns' parameters from row to row
// and has the next row's data on the way while it works on one.
template <typename T, int TPR, int V>
__global__ __launch_bounds__(threads_of(TPR)) void norm_fwd_kernel(NormArgs a) {
    constexpr int E = Chunk<T>::kN, kThreads = threads_of(TPR), kSlots = kThreads / TPR;
    __shared__ f32x2 mem[2][16];
    int turn = 0;
    const int t = threadIdx.x % TPR, slot = threadIdx.x / TPR;
    const float inv = 1.0f / static_cast<float>(a.C);
    const bool single = a.rows_per_gate == 1;

    // sum over the row of f(element)
    auto total = [&](auto f) {
        float s = 0.0f, none = 0.0f;
#pragma unroll
        for (int k = 0; k < V; ++k)
#pragma unroll
            for (int i = 0; i < E; ++i) s = f(s, k, i);
        row_sum<TPR>(s, none, mem, turn);
        return s;
    };
    // deviations from the mean in place, their 1 / sqrt in rstd
    auto norm = [&](float (&v)[V][E], float &mean, float &rstd) {
        mean = 0.0f;
        if (a.layer) {
            mean = total([&](float s, int k, int i) { return s + v[k][i]; }) * inv;
#pragma unroll
            for (int k = 0; k < V; ++k)
#pragma unroll
                for (int i = 0; i < E; ++i) v[k][i] = (k * TPR + t) * E + i < a.C ? v[k][i] - mean : 0.0f;
        }
        rstd = 1.0f / sqrtf(total([&](float s, int k, int i) { return fmaf(v[k][i], v[k][i], s); }) * inv + a.eps);
    };

    float w1[V][E], c1[V][E], w2[V][E], c2[V][E], gate[V][E];
#pragma unroll
    for (int k = 0; k < V; ++k) {
        const int col = (k * TPR + t) * E;
        load_param<E>(a.w1, col, a.C, a.pvec, 1.0f, w1[k]);
        load_param<E>(a.c1, col, a.C, a.pvec, 0.0f, c1[k]);
        load_param<E>(a.w2, col, a.C, a.pvec, 1.0f, w2[k]);
        load_param<E>(a.c2, col, a.C, a.pvec, 0.0f, c2[k]);
#pragma unroll
        for (int i = 0; i < E; ++i) gate[k][i] = a.alpha;
    }
    const int64_t begin = static_cast<int64_t>(blockIdx.x) * a.unit_rows, end = min(begin + a.unit_rows, a.rows);
    // a slot past the last row repeats it and stores nothing
    auto row_of = [&](int64_t first) { return min(first + slot, end - 1); };
    RowChunk<T, V> x = fetch<T, TPR, V>(a.x, row_of(begin), a.x_stride, t, a.C, a.vec), b{};
    if (a.branch) b = fetch<T, TPR, V>(a.branch, row_of(begin), a.b_stride, t, a.C, a.vec);
    uint32_t had = 0xffffffffu;
    for (int64_t first = begin; first < end; first += kSlots) {
        const int64_t r = row_of(first);
        const bool on = first + slot < end;
        float y[V][E], stat[4] = {};
#pragma unroll
        for (int k = 0; k < V; ++k)
#pragma unroll
            for (int i = 0; i < E; ++i) y[k][i] = value(x, k, i);
        if (a.gate) {
            const uint32_t g = single ? static_cast<uint32_t>(r) : fdiv(static_cast<uint32_t>(r), a.gate_div);
            if (g != had) {
                had = g;
#pragma unroll
                for (int k = 0; k < V; ++k) {
                    load_param<E>(a.gate + static_cast<int64_t>(g) * a.C, (k * TPR + t) * E, a.C, a.pvec, 0.0f, gate[k]);
#pragma unroll
                    for (int i = 0; i < E; ++i) gate[k][i] *= a.alpha;
                }
            }
        }
        RowChunk<T, V> nx{}, nb{};
        if (first + kSlots < end) {
            nx = fetch<T, TPR, V>(a.x, row_of(first + kSlots), a.x_stride, t, a.C, a.vec);
            if (a.branch) nb = fetch<T, TPR, V>(a.branch, row_of(first + kSlots), a.b_stride, t, a.C, a.vec);
        }
        if (a.branch) {
            float z[V][E];
#pragma unroll
            for (int k = 0; k < V; ++k)
#pragma unroll
                for (int i = 0; i < E; ++i) z[k][i] = value(b, k, i);
            norm(z, stat[0], stat[1]);
#pragma unroll
            for (int k = 0; k < V; ++k)
#pragma unroll
                for (int i = 0; i < E; ++i) {
                    y[k][i] = fmaf(gate[k][i], fmaf(z[k][i] * stat[1], w1[k][i], c1[k][i]), y[k][i]);
                    if ((k * TPR + t) * E + i >= a.C) y[k][i] = 0.0f;
                }
        }
        if (a.y && on) {
#pragma unroll
            for (int k = 0; k < V; ++k)
                store_row<T, E>(static_cast<T *>(a.y) + r * a.C, (k * TPR + t) * E, a.C, a.vec, y[k]);
        }
        if (a.second) {
            norm(y, stat[2], stat[3]);
#pragma unroll
            for (int k = 0; k < V; ++k) {
#pragma unroll
                for (int i = 0; i < E; ++i) y[k][i] = fmaf(y[k][i] * stat[3], w2[k][i], c2[k][i]);
                if (on && a.u) store_row<T, E>(static_cast<T *>(a.u) + r * a.C, (k * TPR + t) * E, a.C, a.vec, y[k]);
            }
        }
        if (a.stats && t == 0 && on)
            *(REX_GLOBAL f32x4 *)(a.stats + r * 4) = f32x4{stat[0], stat[1], stat[2], stat[3]};
        x = nx;
        b = nb;
    }
}

template <typename T, int TPR, int V>
__global__ __launch_bounds__(threads_of(TPR)) void norm_bwd_kernel(NormArgs a) {
    constexpr int E = Chunk<T>::kN, kThreads = threads_of(TPR), kSlots = kThreads / TPR;
    extern __shared__ float cols[];               // [kSlots][C]
    __shared__ f32x2 mem[2][16];
    int turn = 0;
    const int t = threadIdx.x % TPR, slot = threadIdx.x / TPR;
    const float inv = 1.0f / static_cast<float>(a.C);
    float sw1[V][E] = {}, sc1[V][E] = {}, sw2[V][E] = {}, sc2[V][E] = {}, sg[V][E] = {};
    const bool each = a.gate && a.rows_per_gate == 1;
    float w1[V][E], c1[V][E], w2[V][E], gate[V][E];
#pragma unroll
    for (int k = 0; k < V; ++k) {
        const int col = (k * TPR + t) * E;
        load_param<E>(a.w1, col, a.C, a.pvec, 1.0f, w1[k]);
        load_param<E>(a.c1, col, a.C, a.pvec, 0.0f, c1[k]);
        load_param<E>(a.w2, col, a.C, a.pvec, 1.0f, w2[k]);
#pragma unroll
        for (int i = 0; i < E; ++i) gate[k][i] = 1.0f;
    }

    // sums over the row slots, in order, to dst[C]
    auto flush = [&](const float (&s)[V][E], float *dst) {
        if constexpr (kSlots == 1) {
#pragma unroll
            for (int k = 0; k < V; ++k)
#pragma unroll
                for (int i = 0; i < E; ++i) {
                    const int col = (k * TPR + t) * E + i;
                    if (col < a.C) as_global_mut<float>(dst)[col] = s[k][i];
                }
        } else {
            __syncthreads();
#pragma unroll
            for (int k = 0; k < V; ++k)
#pragma unroll
                for (int i = 0; i < E; ++i) {
                    const int col = (k * TPR + t) * E + i;
                    if (col < a.C) cols[slot * a.C + col] = s[k][i];
                }
            __syncthreads();
            for (int col = threadIdx.x; col < a.C; col += kThreads) {
                float x = 0.0f;
                for (int q = 0; q < kSlots; ++q) x += cols[q * a.C + col];
                as_global_mut<float>(dst)[col] = x;
            }
        }
    };

    for (int64_t unit = blockIdx.x; unit < a.units; unit += a.blocks) {
        const int64_t seg = unit / a.gate_parts, in = (unit - seg * a.gate_parts) * a.unit_rows;
        const int64_t begin = seg * a.span + in;
        const int64_t end = min(min(begin + a.unit_rows, (seg + 1) * a.span), a.rows);
        auto row_of = [&](int64_t first) { return min(first + slot, end - 1); };
        auto load_gate = [&](int64_t g) {
#pragma unroll
            for (int k = 0; k < V; ++k)
                load_param<E>(a.gate + g * a.C, (k * TPR + t) * E, a.C, a.pvec, 0.0f, gate[k]);
        };
        if (a.gate && !each) load_gate(seg);
        RowChunk<T, V> x{}, b{}, gu{}, gy{};
        auto fetch_all = [&](int64_t r) {
            x = fetch<T, TPR, V>(a.x, r, a.x_stride, t, a.C, a.vec);
            if (a.branch) b = fetch<T, TPR, V>(a.branch, r, a.b_stride, t, a.C, a.vec);
            if (a.gu) gu = fetch<T, TPR, V>(a.gu, r, a.C, t, a.C, a.vec);
            if (a.gy) gy = fetch<T, TPR, V>(a.gy, r, a.C, t, a.C, a.vec);
        };
        if (begin < end) fetch_all(row_of(begin));
        for (int64_t first = begin; first < end; first += kSlots) {
            const bool on = first + slot < end;
            const int64_t r = row_of(first);
            const f32x4 st = *(const REX_GLOBAL f32x4 *)(a.stats + r * 4);
            if (each) load_gate(r);
            // hat1: N1's normalised row; y: N2's, from y = x + alpha gate N1(branch); d: the
            // gradient of y, g: upstream gradients times weights
            float hat1[V][E], y[V][E], d[V][E], g[V][E];
            float s1 = 0.0f, s0 = 0.0f;
#pragma unroll
            for (int k = 0; k < V; ++k)
#pragma unroll
                for (int i = 0; i < E; ++i) {
                    hat1[k][i] = (value(b, k, i) - st[0]) * st[1];
                    y[k][i] = value(x, k, i);
                    if (a.branch)
                        y[k][i] = fmaf(a.alpha * gate[k][i], fmaf(hat1[k][i], w1[k][i], c1[k][i]), y[k][i]);
                    y[k][i] = (y[k][i] - st[2]) * st[3];
                    const float u = value(gu, k, i);
                    if (on) {
                        sw2[k][i] = fmaf(u, y[k][i], sw2[k][i]);
                        sc2[k][i] += u;
                    }
                    g[k][i] = u * w2[k][i];              // 0 past C, as u
                    s1 = fmaf(g[k][i], y[k][i], s1);
                    s0 += g[k][i];
                    d[k][i] = value(gy, k, i);
                }
            if (first + kSlots < end) fetch_all(row_of(first + kSlots));
            if (a.gu) {
                row_sum<TPR>(s1, s0, mem, turn);
                s1 *= inv;
                s0 = a.layer ? s0 * inv : 0.0f;
#pragma unroll
                for (int k = 0; k < V; ++k)
#pragma unroll
                    for (int i = 0; i < E; ++i) d[k][i] += st[3] * ((g[k][i] - s0) - y[k][i] * s1);
            }
            if (on && a.gx) {
#pragma unroll
                for (int k = 0; k < V; ++k)
                    store_row<T, E>(static_cast<T *>(a.gx) + r * a.C, (k * TPR + t) * E, a.C, a.vec, d[k]);
            }
            if (!a.branch) continue;
            float m1 = 0.0f, m0 = 0.0f;
#pragma unroll
            for (int k = 0; k < V; ++k)
#pragma unroll
                for (int i = 0; i < E; ++i) {
                    const int col = (k * TPR + t) * E + i;
                    const float ad = col < a.C ? a.alpha * d[k][i] : 0.0f;
                    const float gz = gate[k][i] * ad, dg = ad * fmaf(hat1[k][i], w1[k][i], c1[k][i]);
                    if (on) {
                        sg[k][i] += dg;
                        sw1[k][i] = fmaf(gz, hat1[k][i], sw1[k][i]);
                        sc1[k][i] += gz;
                        if (each && a.ggate && col < a.C) as_global_mut<float>(a.ggate)[r * a.C + col] = dg;
                    }
                    g[k][i] = gz * w1[k][i];
                    m1 = fmaf(g[k][i], hat1[k][i], m1);
                    m0 += g[k][i];
                }
            row_sum<TPR>(m1, m0, mem, turn);
            m1 *= inv;
            m0 = a.layer ? m0 * inv : 0.0f;
            if (on && a.gb) {
#pragma unroll
                for (int k = 0; k < V; ++k) {
                    float e[E];
#pragma unroll
                    for (int i = 0; i < E; ++i) e[i] = st[1] * ((g[k][i] - m0) - hat1[k][i] * m1);
                    store_row<T, E>(static_cast<T *>(a.gb) + r * a.C, (k * TPR + t) * E, a.C, a.vec, e);
                }
            }
        }
        if (a.gate_sum) {
            flush(sg, a.gate_part + unit * a.C);
#pragma unroll
            for (int k = 0; k < V; ++k)
#pragma unroll
                for (int i = 0; i < E; ++i) sg[k][i] = 0.0f;
        }
    }
    float *dst = a.part + static_cast<int64_t>(blockIdx.x) * 4 * a.C;
    if (a.gw1) flush(sw1, dst);
    if (a.gc1) flush(sc1, dst + a.C);
    if (a.gw2) flush(sw2, dst + 2 * a.C);
    if (a.gc2) flush(sc2, dst + 3 * a.C);
}

// Column sums of the partial rows: 64 columns, 16 slices of the rows side by side, in order.
// blockIdx.y: 0..3 the four parameters, 4 + g the gate row g.
__global__ __launch_bounds__(1024) void norm_columns_kernel(NormArgs a, int gates_first) {
    __shared__ float part[16][64];
    const int col = blockIdx.x * 64 + (threadIdx.x & 63), slice = threadIdx.x >> 6;
    const int64_t which = static_cast<int64_t>(blockIdx.y) + gates_first;
    const float *src;
    float *dst;
    int64_t n, step;
    if (which < 4) {
        dst = which == 0 ? a.gw1 : which == 1 ? a.gc1 : which == 2 ? a.gw2 : a.gc2;
        src = a.part + which * a.C;
        n = a.blocks;
        step = 4 * static_cast<int64_t>(a.C);
    } else {
        dst = a.ggate + (which - 4) * a.C;
        src = a.gate_part + (which - 4) * a.gate_parts * a.C;
        n = a.gate_parts;
        step = a.C;
    }
    if (!dst) return;                             // the whole workgroup
    float s = 0.0f;
    if (col < a.C) {
        // eight loads on their way at once: one after the other 32 of them took 10 us
#pragma unroll 8
        for (int64_t i = slice; i < n; i += 16) s += as_global<float>(src)[i * step + col];
    }
    part[slice][threadIdx.x & 63] = s;
    __syncthreads();
    if (slice == 0 && col < a.C) {
        for (int q = 1; q < 16; ++q) s += part[q][threadIdx.x];
        as_global_mut<float>(dst)[col] = s;
    }
}

template <typename T, int TPR, int V>
void run_fwd(const NormArgs &a, hipStream_t s) {
    hipLaunchKernelGGL((norm_fwd_kernel<T, TPR, V>), dim3(a.blocks), dim3(threads_of(TPR)), 0, s, a);
}
template <typename T, int TPR, int V>
void run_bwd(const NormArgs &a, hipStream_t s) {
    constexpr int kThreads = threads_of(TPR);
    constexpr int kSlots = kThreads / TPR;
    const size_t lds = kSlots > 1 ? static_cast<size_t>(kSlots) * a.C * 4 : 0;
    if (a.blocks > 0)
        hipLaunchKernelGGL((norm_bwd_kernel<T, TPR, V>), dim3(a.blocks), dim3(kThreads), lds, s, a);
}

// Threads of a row by its chunks of 16 bytes: one chunk a thread, so that the backward's five
// column sums fit the registers, and two for rows that 1024 threads do not cover.
template <typename T, bool BWD>
void run_sized(const NormArgs &a, hipStream_t s) {
    const int chunks = (a.C + Chunk<T>::kN - 1) / Chunk<T>::kN;
#define REX_NORM(TPR, V)                      \
    do {                                      \
        if (BWD) run_bwd<T, TPR, V>(a, s);    \
        else run_fwd<T, TPR, V>(a, s);        \
        return;                               \
    } while (0)
    if (chunks <= 16) REX_NORM(16, 1);
    if (chunks <= 32) REX_NORM(32, 1);
    if (chunks <= 64) REX_NORM(64, 1);
    if (chunks <= 128) REX_NORM(128, 1);
    if (chunks <= 256) REX_NORM(256, 1);
    if (chunks <= 512) REX_NORM(512, 1);
    if (chunks <= 1024) REX_NORM(1024, 1);
    if constexpr (sizeof(T) == 4) REX_NORM(1024, 2);
#undef REX_NORM
}

}  // namespace

int norm_slots(int dtype, int C) {
    const int chunks = (C + (dtype == kBF16 ? 7 : 3)) / (dtype == kBF16 ? 8 : 4);
    return chunks <= 16 ? 16 : chunks <= 32 ? 8 : chunks <= 64 ? 4 : chunks <= 128 ? 2 : 1;
}

hipError_t launch_norm_fwd(const NormArgs &a, int dtype, hipStream_t s) {
    if (dtype == kBF16) run_sized<uint16_t, false>(a, s);
    else run_sized<float, false>(a, s);
    return hipGetLastError();
}

hipError_t launch_norm_bwd(const NormArgs &a, int dtype, hipStream_t s) {
    if (dtype == kBF16) run_sized<uint16_t, true>(a, s);
    else run_sized<float, true>(a, s);
    const int cols = (a.C + 63) / 64;
    const bool params = a.gw1 || a.gc1 || a.gw2 || a.gc2;
    const bool gates = a.gate_sum != 0;
    // one launch for parameters and gate rows; more gate rows than a grid has go in turns
    int64_t from = params ? 0 : 4, to = gates ? 4 + a.gates : 4;
    for (; from < to; from += 65535)
        hipLaunchKernelGGL(norm_columns_kernel,
                           dim3(cols, static_cast<uint32_t>(to - from < 65535 ? to - from : 65535)),
                           dim3(1024), 0, s, a, static_cast<int>(from));
    return hipGetLastError();
}

}  // namespace rex
