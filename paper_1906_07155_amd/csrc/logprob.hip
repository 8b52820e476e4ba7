// logprob.hip -- log probabilities of classes, their entropy, the top classes, and the gradient.
//
// A row's logits are read once and stay in registers: 16 lanes, a wave or a workgroup hold a row, or
// a part of a long one (whose parts a second kernel joins).  The entropy comes from the same sums:
// with d = x - max x, s = sum exp(d) and t = sum d exp(d), it is log s - t / s, two terms of one sign.
// The top classes are found one after the other, as the largest of 64-bit keys: the logit's bits in
// the order of the numbers, then the class, the lower one first.
//
// Rows begin at any element: a lane's 16 bytes are at a multiple of 16 all the same, and what is not of the
// row counts as -inf (from the row's first element on, 32768 rows of 1231 bf16 took 32 us instead of 26).
// What bounds it is memory: the
// gradient needs the sums of the whole row, so that training reads the logits twice.  4096 rows of 32000 in bf16
// 74 us (3.5 TB/s) and 108 (4.9 TB/s), 8192 of 1231, which caches hold, 11 and 13.  Few rows are bound by their steps,
// each of which needs the one before: 16 of 100003 in binary32, with their eight top classes, 12 us in 25 parts
// each and 6 for the joining.
#include "logprob.hpp"
#include "attn.hpp"

namespace rex {

namespace {

template <typename T> struct Chunk {
    static constexpr int kN = 16 / sizeof(T);
    using V = T __attribute__((ext_vector_type(kN), aligned(sizeof(T))));
};

// Elements at .. at + kN - 1 of a row of n, `none` where there is no such element: 16 bytes at a multiple of
// 16, which may hold elements beside the row (of other rows, or between them), as long as they lie between
// the first row's first element and the last row's last.
struct Bounds {
    const char *low, *high;
};
template <typename T>
__device__ __forceinline__ void load_chunk(const T *row, int at, int n, const Bounds &b, float none, float *x) {
    constexpr int kN = Chunk<T>::kN;
    using V = typename Chunk<T>::V;
    if (at >= n) {
#pragma unroll
        for (int i = 0; i < kN; ++i) x[i] = none;
        return;
    }
    const char *p = reinterpret_cast<const char *>(row + at);
    if (p >= b.low && p + 16 <= b.high) {
        const V v = *(const REX_GLOBAL V *)(p);
#pragma unroll
        for (int i = 0; i < kN; ++i) {
            if constexpr (sizeof(T) == 2) x[i] = bf16_to_f32(v[i]);
            else x[i] = v[i];
        }
        if (at < 0 || at + kN > n) {
#pragma unroll
            for (int i = 0; i < kN; ++i) x[i] = at + i >= 0 && at + i < n ? x[i] : none;
        }
    } else {
#pragma unroll
        for (int i = 0; i < kN; ++i)
            x[i] = at + i >= 0 && at + i < n ? load_f32<T>(as_global<T>(row) + at + i) : none;
    }
}
template <typename T>
__device__ __forceinline__ void store_chunk(T *row, int at, int n, const float *x) {
    constexpr int kN = Chunk<T>::kN;
    using V = typename Chunk<T>::V;
    if (at >= 0 && at + kN <= n) {
        V v;
#pragma unroll
        for (int i = 0; i < kN; ++i) {
            if constexpr (sizeof(T) == 2) v[i] = __builtin_bit_cast(uint16_t, static_cast<__bf16>(x[i]));
            else v[i] = x[i];
        }
        *(REX_GLOBAL V *)(row + at) = v;
    } else {
#pragma unroll
        for (int i = 0; i < kN; ++i)
            if (at + i >= 0 && at + i < n) store_f32<T>(as_global_mut<T>(row) + at + i, x[i]);
    }
}
// How many elements of its 16 bytes come before a row.
template <typename T> __device__ __forceinline__ int lead_of(const T *row) {
    return static_cast<int>(reinterpret_cast<uintptr_t>(row) / sizeof(T)) & (Chunk<T>::kN - 1);
}
template <typename T> __device__ __forceinline__ Bounds bounds_of(const LogprobArgs &a) {
    const T *p = static_cast<const T *>(a.logits);
    return Bounds{reinterpret_cast<const char *>(p), reinterpret_cast<const char *>(p + (a.rows - 1) * a.stride + a.C)};
}

// The bits of x in the order of the numbers, NaN above all; never 0.
__device__ __forceinline__ uint32_t ordered(float x) {
    const uint32_t b = __float_as_uint(x + 0.0f);              // (-0 is 0)
    return x != x ? 0xffffffffu : b ^ (static_cast<int32_t>(b) < 0 ? 0xffffffffu : 0x80000000u);
}
__device__ __forceinline__ uint64_t make_key(uint32_t value, int c) {
    return static_cast<uint64_t>(value) << 32 | (0xfffffffeu - static_cast<uint32_t>(c));      // (never all ones)
}
__device__ __forceinline__ float key_value(uint64_t k) {
    const uint32_t b = static_cast<uint32_t>(k >> 32);
    return b == 0xffffffffu ? __builtin_nanf("") : __uint_as_float(b ^ (b >> 31 ? 0x80000000u : 0xffffffffu));
}
__device__ __forceinline__ int key_class(uint64_t k) { return static_cast<int>(0xfffffffeu - static_cast<uint32_t>(k)); }

// over the `LANES` lanes of a row
template <int LANES> __device__ __forceinline__ float lanes_max(float x) {
#pragma unroll
    for (int d = LANES / 2; d > 0; d /= 2) x = fmaxf(x, __shfl_xor(x, d));
    return x;
}
template <int LANES> __device__ __forceinline__ float lanes_sum(float x) {
#pragma unroll
    for (int d = LANES / 2; d > 0; d /= 2) x += __shfl_xor(x, d);
    return x;
}
template <int LANES> __device__ __forceinline__ uint64_t lanes_max(uint64_t x) {
#pragma unroll
    for (int d = LANES / 2; d > 0; d /= 2) {
        const uint64_t y = __shfl_xor(static_cast<unsigned long long>(x), d);
        x = y > x ? y : x;
    }
    return x;
}

__device__ __forceinline__ void add_part(LogPart &a, const LogPart &b) {
    const float top = fmaxf(a.top, b.top), from = top == -kInf ? 0.0f : top;
    // (a part without a class has sum 0)
    const float da = a.top == -kInf ? 0.0f : a.top - from, db = b.top == -kInf ? 0.0f : b.top - from;
    const float ea = __builtin_amdgcn_exp2f(da * kLog2e), eb = __builtin_amdgcn_exp2f(db * kLog2e);
    // (a part far below the other adds nothing: its distance may be past the finite numbers)
    a.moment = (ea == 0.0f ? 0.0f : (a.moment + da * a.sum) * ea) + (eb == 0.0f ? 0.0f : (b.moment + db * b.sum) * eb);
    a.sum = a.sum * ea + b.sum * eb;
    a.top = top;
}

constexpr float kLn2 = 0.69314718055994531f;

// A row's results.  The log sum is relative to the largest x, and both stay apart in the results: their
// sum would be rounded at the size of x, and a row all of whose logits are at -1e9 has the probabilities
// that it has with all of them at 0.
struct RowStats {
    float top, log_sum;
};
__device__ __forceinline__ float log_prob(const RowStats &r, float x) {
    return r.top == -kInf ? -kInf : (x - r.top) - r.log_sum;
}
__device__ __forceinline__ RowStats row_stats(const LogPart &p) {
    const bool none = p.sum == 0.0f;
    // (the largest of nothing but NaN, or NaN and -inf, is -inf: their sum tells)
    return RowStats{none ? -kInf : p.sum != p.sum ? p.sum : p.top, none ? 0.0f : __builtin_amdgcn_logf(p.sum) * kLn2};
}
// The label's x, if it is counted.
struct Label {
    float x;
    bool counted;
};
template <typename T> __device__ __forceinline__ Label load_label(const LogprobArgs &a, int64_t row) {
    const int64_t c = as_global<int64_t>(a.labels)[row];
    const bool counted = c >= 0 && c < a.C;
    return Label{counted ? a.scale * load_f32<T>(as_global<T>(a.logits) + row * a.stride + c) : 0.0f, counted};
}
__device__ __forceinline__ void store_row(const LogprobArgs &a, int64_t row, const LogPart &p, const RowStats &r, const Label &l) {
    as_global_mut<float>(a.logp)[row] = l.counted ? log_prob(r, l.x) : 0.0f;
    as_global_mut<float>(a.entropy)[row] = p.sum == 0.0f ? 0.0f : r.log_sum - p.moment / p.sum;
    *(REX_GLOBAL f32x2 *)(a.stats + 2 * row) = f32x2{r.top, r.log_sum};
}
__device__ __forceinline__ void store_top(const LogprobArgs &a, int64_t row, int i, uint64_t key, const RowStats &r) {
    as_global_mut<float>(a.top_logp)[row * a.top + i] = log_prob(r, a.scale * key_value(key));
    as_global_mut<int64_t>(a.top_index)[row * a.top + i] = key_class(key);
}

// LANES lanes (of a wave, or a workgroup of four waves) hold a part of a row in N chunks each.
template <typename T, int LANES, int N>
__global__ __launch_bounds__(256) void logprob_fwd_kernel(LogprobArgs a) {
    constexpr int kN = Chunk<T>::kN, kRows = 256 / LANES, kIn = LANES < 64 ? LANES : 64;
    constexpr int kWaves = LANES / kIn;
    __shared__ LogPart parts[4];
    __shared__ uint64_t best[2][4];
    const int lane = threadIdx.x % LANES, wave = threadIdx.x / 64;
    const int64_t item = blockIdx.x * int64_t(kRows) + threadIdx.x / LANES;
    const int64_t row = item / a.parts;
    if (row >= a.rows) return;                      // (a whole workgroup, where it shares a row)
    const int part = static_cast<int>(item % a.parts), first = part * a.each;
    const int n = min(a.each, a.C - first);
    const T *from = static_cast<const T *>(a.logits) + row * a.stride + first;

    const int lead = lead_of(from);
    const Bounds bounds = bounds_of<T>(a);
    float x[N * kN];
#pragma unroll
    for (int i = 0; i < N; ++i) load_chunk<T>(from, (i * LANES + lane) * kN - lead, n, bounds, -kInf, x + i * kN);
    Label label{};
    if (a.parts == 1) label = load_label<T>(a, row);
    // (the logits themselves are what is ordered: a scale may round two of them to one number)
    uint32_t v[N * kN];
    if (a.top > 0) {
#pragma unroll
        for (int i = 0; i < N * kN; ++i) {
            const int at = (i / kN * LANES + lane) * kN + i % kN - lead;
            v[i] = at >= 0 && at < n ? ordered(x[i]) : 0u;
        }
    }
    LogPart p{-kInf, 0.0f, 0.0f};
#pragma unroll
    for (int i = 0; i < N * kN; ++i) {
        x[i] *= a.scale;
        p.top = fmaxf(p.top, x[i]);
    }
    p.top = lanes_max<kIn>(p.top);
    const float low = p.top == -kInf ? 0.0f : p.top;
#pragma unroll
    for (int i = 0; i < N * kN; ++i) {
        const float d = x[i] - low, e = __builtin_amdgcn_exp2f(d * kLog2e);
        p.sum += e;
        p.moment = fmaf(fmaxf(d, -3e38f), e, p.moment);      // (0 for what is at -inf)
    }
    p.sum = lanes_sum<kIn>(p.sum);
    p.moment = lanes_sum<kIn>(p.moment);
    if constexpr (kWaves > 1) {
        if ((threadIdx.x & 63) == 0) parts[wave] = p;
        __syncthreads();
        p = parts[0];
#pragma unroll
        for (int w = 1; w < kWaves; ++w) add_part(p, parts[w]);
    }
    const RowStats stats = row_stats(p);
    if (lane == 0) {
        if (a.parts > 1) a.part[row * a.parts + part] = p;
        else store_row(a, row, p, stats, label);
    }
    if (a.top == 0) return;
    uint64_t found = 0;                            // of lane r: the r-th

    for (int r = 0; r < a.top; ++r) {
        uint32_t most = 0;
        int at = 0;
#pragma unroll
        for (int i = 0; i < N * kN; ++i)
            if (v[i] > most) {
                most = v[i];
                at = i;
            }
        const uint64_t mine = most ? make_key(most, first + (at / kN * LANES + lane) * kN + at % kN - lead) : 0;
        uint64_t key = lanes_max<kIn>(mine);
        if constexpr (kWaves > 1) {
            if ((threadIdx.x & 63) == 0) best[r & 1][wave] = key;
            __syncthreads();
#pragma unroll
            for (int w = 0; w < kWaves; ++w) key = best[r & 1][w] > key ? best[r & 1][w] : key;
        }
#pragma unroll
        for (int i = 0; i < N * kN; ++i)
            if (mine == key && i == at) v[i] = 0;
        found = lane == r ? key : found;
    }
    if (lane >= a.top) return;
    if (a.parts > 1) a.keys[(row * a.parts + part) * a.top + lane] = found;
    else store_top(a, row, lane, found, stats);
}

// A wave for each row, over its parts.
template <typename T>
__global__ __launch_bounds__(64) void logprob_join_kernel(LogprobArgs a) {
    const int64_t row = blockIdx.x;
    const int lane = threadIdx.x;
    constexpr int kKeys = 4;                         // of a lane, in registers
    const uint64_t *keys = a.keys + row * a.parts * a.top;
    uint64_t held[kKeys];
#pragma unroll
    for (int i = 0; i < kKeys; ++i) held[i] = 64 * i + lane < a.parts * a.top ? as_global<uint64_t>(keys)[64 * i + lane] : 0;
    const Label label = load_label<T>(a, row);
    LogPart p{-kInf, 0.0f, 0.0f};
    for (int i = lane; i < a.parts; i += 64) add_part(p, a.part[row * a.parts + i]);
#pragma unroll
    for (int d = 32; d > 0; d /= 2) {
        const LogPart q{__shfl_xor(p.top, d), __shfl_xor(p.sum, d), __shfl_xor(p.moment, d)};
        // (both lanes of a pair add in one order)
        LogPart lo = lane & d ? q : p;
        add_part(lo, lane & d ? p : q);
        p = lo;
    }
    const RowStats stats = row_stats(p);
    if (lane == 0) store_row(a, row, p, stats, label);
    if (a.top == 0) return;
    const int count = a.parts * a.top;
    uint64_t last = ~uint64_t(0), found = 0;
    for (int r = 0; r < a.top; ++r) {                // the largest of those below the last one
        uint64_t key = 0;
        const auto look = [&](uint64_t k) { key = k < last && k > key ? k : key; };
#pragma unroll
        for (int i = 0; i < kKeys; ++i) look(held[i]);
        for (int i = 64 * kKeys + lane; i < count; i += 64) look(as_global<uint64_t>(keys)[i]);
        last = lanes_max<64>(key);
        found = lane == r ? last : found;
    }
    if (lane < a.top) store_top(a, row, lane, found, stats);
}

template <typename T, int LANES, int N>
__global__ __launch_bounds__(256) void logprob_bwd_kernel(LogprobArgs a) {
    constexpr int kN = Chunk<T>::kN, kRows = 256 / LANES;
    const int lane = threadIdx.x % LANES;
    const int64_t item = blockIdx.x * int64_t(kRows) + threadIdx.x / LANES;
    const int64_t row = item / a.parts;
    if (row >= a.rows) return;
    const int first = static_cast<int>(item % a.parts) * a.each, n = min(a.each, a.C - first);
    const T *from = static_cast<const T *>(a.logits) + row * a.stride + first;
    T *to = static_cast<T *>(a.grad) + row * a.C + first;
    const int64_t label = as_global<int64_t>(a.labels)[row];
    const bool counted = label >= 0 && label < a.C;
    const f32x2 held = *(const REX_GLOBAL f32x2 *)(a.stats + 2 * row);
    const RowStats stats{held[0], held[1]};
    const float entropy = as_global<float>(a.entropy)[row];
    const float gl = a.glogp && counted ? as_global<float>(a.glogp)[row] : 0.0f;
    const float gh = a.gentropy ? as_global<float>(a.gentropy)[row] : 0.0f;
    const int at_label = counted ? static_cast<int>(label) - first : -1;
    const int lead = lead_of(from);
    const Bounds bounds = bounds_of<T>(a);
    float x[N * kN];
#pragma unroll
    for (int i = 0; i < N; ++i) load_chunk<T>(from, (i * LANES + lane) * kN - lead, n, bounds, -kInf, x + i * kN);
#pragma unroll
    for (int i = 0; i < N; ++i) {
        const int at = (i * LANES + lane) * kN - lead;
#pragma unroll
        for (int j = 0; j < kN; ++j) {
            const float logs = log_prob(stats, a.scale * x[i * kN + j]);
            const float p = __builtin_amdgcn_exp2f(logs * kLog2e);
            float g = p == 0.0f ? 0.0f : -p * fmaf(gh, logs + entropy, gl);
            if (at + j == at_label) g += gl;
            x[i * kN + j] = stats.top == -kInf ? 0.0f : a.scale * g;
        }
        if (at < n) store_chunk<T>(to, at, n, x + i * kN);
    }
}

// How many lanes hold a row or part, and in how many chunks.
template <template <typename, int, int> class Launch, typename T>
hipError_t choose(const LogprobArgs &a, hipStream_t s) {
    constexpr int kN = Chunk<T>::kN;
    // a row that may begin between multiples of 16 bytes takes a chunk more
    const bool even = reinterpret_cast<uintptr_t>(a.logits) % 16 == 0 && a.stride % kN == 0 && a.each % kN == 0;
    const int need = a.each + (even ? 0 : kN - 1);
    if (need <= 16 * kN) return Launch<T, 16, 1>::run(a, s);
    if (need <= 64 * kN) return Launch<T, 64, 1>::run(a, s);
    if (need <= 128 * kN) return Launch<T, 64, 2>::run(a, s);
    if (need <= 192 * kN) return Launch<T, 64, 3>::run(a, s);
    if (need <= 256 * kN) return Launch<T, 64, 4>::run(a, s);
    if constexpr (kN < 8) {
        if (need <= 512 * kN) return Launch<T, 256, 2>::run(a, s);
        if (need <= 768 * kN) return Launch<T, 256, 3>::run(a, s);
    }
    return Launch<T, 256, kLogprobRegisters / 256 / kN>::run(a, s);
}
template <typename T, int LANES, int N> struct Forward {
    static hipError_t run(const LogprobArgs &a, hipStream_t s) {
        const int64_t items = a.rows * a.parts;
        logprob_fwd_kernel<T, LANES, N><<<static_cast<uint32_t>((items * LANES + 255) / 256), 256, 0, s>>>(a);
        return hipGetLastError();
    }
};
template <typename T, int LANES, int N> struct Backward {
    static hipError_t run(const LogprobArgs &a, hipStream_t s) {
        const int64_t items = a.rows * a.parts;
        logprob_bwd_kernel<T, LANES, N><<<static_cast<uint32_t>((items * LANES + 255) / 256), 256, 0, s>>>(a);
        return hipGetLastError();
    }
};

}  // namespace

hipError_t launch_logprob_fwd(const LogprobArgs &a, int dtype, hipStream_t s) {
    const hipError_t e = dtype == kBF16 ? choose<Forward, uint16_t>(a, s) : choose<Forward, float>(a, s);
    if (e != hipSuccess || a.parts == 1) return e;
    if (dtype == kBF16) logprob_join_kernel<uint16_t><<<static_cast<uint32_t>(a.rows), 64, 0, s>>>(a);
    else logprob_join_kernel<float><<<static_cast<uint32_t>(a.rows), 64, 0, s>>>(a);
    return hipGetLastError();
}

hipError_t launch_logprob_bwd(const LogprobArgs &a, int dtype, hipStream_t s) {
    return dtype == kBF16 ? choose<Backward, uint16_t>(a, s) : choose<Backward, float>(a, s);
}

}  // namespace rex
