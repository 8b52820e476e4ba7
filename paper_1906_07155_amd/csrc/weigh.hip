// weigh.hip -- the attention that each remembered box has received (box_memory_weigh).
//
// The logits are made as in the recall (attn_fwd.hpp): keys are the rows of the products and queries
// their columns, so a lane has eight keys of one query, and adds their weights up over heads and
// queries in its registers; the sixteen lanes of a row meet at the end, once for a page.  Sums over
// keys are not needed, the log sum is given, and so nothing but half of the memory is read: codes and
// scales of the keys, and the boxes.
//
// Few queries of a stream (at most 16): a wave takes a page, all of its heads, several heads' codes on
// their way at once; memory bounds it.  More: a workgroup takes a page, its waves share heads and
// queries out, and the buckets of 256 queries against the page's boxes are computed once for all heads
// into LDS; vector instructions bound it.
#include "attn.hpp"
#include "evict.hpp"

namespace rex {

namespace {

// One head's keys of a page: codes and scales as they lie in memory.
template <int DB> struct KeyCodes {
    u32x2 c[2][DB];
    f32x4 s[2];
};
template <int DB>
__device__ __forceinline__ void load_codes(const AttnArgs &a, int64_t head, const uint32_t (&off)[DB], int g,
                                           KeyCodes<DB> &x) {
    const auto r = make_rsrc(a.mk + head * kTile * a.D, kTile * a.D);
#pragma unroll
    for (int t = 0; t < 2; ++t) {
        x.s[t] = *(const REX_GLOBAL f32x4 *)(a.mks + head * kTile + 8 * g + 4 * t);
#pragma unroll
        for (int k = 0; k < DB; ++k) x.c[t][k] = __builtin_amdgcn_raw_buffer_load_b64(r, off[k], 4 * t * a.D, 0);
    }
}
template <int DB> __device__ __forceinline__ void code_offsets(int D, int n, int g, uint32_t (&off)[DB]) {
#pragma unroll
    for (int k = 0; k < DB; ++k) off[k] = 32 * k + 8 * g < D ? (8 * (n >> 2) + (n & 3)) * D + 32 * k + 8 * g : kBufOOB;
}
template <typename T, int DB>
__device__ __forceinline__ void widen_codes(const KeyCodes<DB> &x, typename Num<T>::Frag (&f)[2][DB]) {
#pragma unroll
    for (int t = 0; t < 2; ++t)
#pragma unroll
        for (int k = 0; k < DB; ++k) {
            Num<T>::widen(f[t][k], 0, x.c[t][k][0]);
            Num<T>::widen(f[t][k], 4, x.c[t][k][1]);
        }
}

// Adds a column's weights of eight keys; bias by key, natural units.
template <typename T, int DB>
__device__ __forceinline__ void add_weights(const typename Num<T>::Frag (&kf)[2][DB], const f32x4 (&ks)[2],
                                            const typename Num<T>::Frag (&q)[DB], const f32x4 (&bias)[2], float scale,
                                            float lse, bool on, float (&sum)[8]) {
    f32x4 x[2] = {};
#pragma unroll
    for (int t = 0; t < 2; ++t)
#pragma unroll
        for (int k = 0; k < DB; ++k) x[t] = Num<T>::mma(kf[t][k], q[k], x[t]);
#pragma unroll
    for (int j = 0; j < 8; ++j) {
        const float s = fmaf(x[j >> 2][j & 3], ks[j >> 2][j & 3] * scale, bias[j >> 2][j & 3]);
        const float p = __builtin_amdgcn_exp2f(fminf(s - lse, 0.0f) * kLog2e);
        sum[j] += on ? p : 0.0f;
    }
}

__device__ __forceinline__ void sum_columns(float (&sum)[8]) {
#pragma unroll
    for (int j = 0; j < 8; ++j)
#pragma unroll
        for (int d = 1; d < 16; d *= 2) sum[j] += __shfl_xor(sum[j], d);
}
// The place's old weight and its new share (lanes 0 .. 31 of a wave: place r of the page).
__device__ __forceinline__ void store_weight(const WeighArgs &w, int b, int tile, int r, int klen, bool there, float x) {
    const int64_t at = (static_cast<int64_t>(b) * w.a.max_pages + tile) * kTile + r;
    const bool on = there && tile * kTile + r < klen;
    const float old = on && w.weight ? w.decay * as_global<float>(w.weight)[at] : 0.0f;
    as_global_mut<float>(w.out)[at] = on ? old + x : 0.0f;
}

constexpr int kFewWaves = 4;

template <typename T, int DB, bool BIAS>
__global__ __launch_bounds__(kFewWaves * 64) void weigh_few_kernel(WeighArgs w) {
    using N = Num<T>;
    using Frag = typename N::Frag;
    constexpr int kHeads = DB == 1 ? 4 : DB == 2 ? 2 : 1;      // whose codes are on their way together
    const AttnArgs &a = w.a;
    const int lane = threadIdx.x & 63, n = lane & 15, g = lane >> 4;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int64_t id = static_cast<int64_t>(blockIdx.x) * kFewWaves + wave;
    if (id >= static_cast<int64_t>(a.B) * a.max_pages) return;
    const int b = static_cast<int>(id / a.max_pages), tile = static_cast<int>(id % a.max_pages);
    const int klen = min(max(a.klen[b], 0), a.Nk), qlen = a.qlen ? min(max(a.qlen[b], 0), a.Nq) : a.Nq;
    const int page = tile * kTile < klen ? as_global<int32_t>(a.pages)[id] : -1;
    const bool there = page >= 0 && page < a.num_pages;
    float sum[8] = {};
    if (there && qlen > 0) {
        uint32_t at[8];                     // byte offsets into a head's table
        if (BIAS) {
            float kx, ky;
            box_centre(*(const REX_GLOBAL f32x4 *)(a.mbox + (static_cast<int64_t>(page) * kTile + (lane & 31)) * 4), kx, ky);
            const BoxGeo geo = box_geo(box_load(a.qbox + b * a.qbox_sb + min(n, qlen - 1) * a.qbox_sr));
#pragma unroll
            for (int j = 0; j < 8; ++j) at[j] = pair_bucket(geo, __shfl(kx, 8 * g + j), __shfl(ky, 8 * g + j), a.rule);
        }
        uint32_t off[DB];
        code_offsets<DB>(a.D, n, g, off);
        for (int first = 0; first < a.Hkv; first += kHeads) {
            KeyCodes<DB> codes[kHeads];
#pragma unroll
            for (int i = 0; i < kHeads; ++i)
                load_codes<DB>(a, static_cast<int64_t>(page) * a.Hkv + min(first + i, a.Hkv - 1), off, g, codes[i]);
            for (int of = 0; of < a.group; ++of) {
                Frag q[kHeads][DB];
                f32x4 bias[kHeads][2];
                float lse[kHeads];
#pragma unroll
                for (int i = 0; i < kHeads; ++i) {
                    const int h = min(first + i, a.Hkv - 1) * a.group + of;
                    const HeadRows qr = head_rows<T>(a.q, b, h, qlen, a.D);
                    Frag x[1][DB];
                    load_columns<T, DB, 1>(qr.at(0), qr.sr, n, g, a.D, x);
#pragma unroll
                    for (int k = 0; k < DB; ++k) q[i][k] = x[0][k];
                    lse[i] = as_global<float>(w.lse)[(static_cast<int64_t>(b) * a.H + h) * a.Nq + min(n, qlen - 1)];
                    bias[i][0] = bias[i][1] = f32x4{};
                    if (BIAS && n < qlen) {
                        const float *table = a.bias + static_cast<int64_t>(h) * a.rule.nb * a.rule.nb;
#pragma unroll
                        for (int j = 0; j < 8; ++j) bias[i][j >> 2][j & 3] = wide_entry(table, at[j]);
                    }
                }
#pragma unroll
                for (int i = 0; i < kHeads; ++i) {
                    Frag kf[2][DB];
                    widen_codes<T, DB>(codes[i], kf);
                    const bool on = n < qlen && first + i < a.Hkv && fabsf(lse[i]) < kInf;
                    add_weights<T, DB>(kf, codes[i].s, q[i], bias[i], a.scale, lse[i], on, sum);
                }
            }
        }
        sum_columns(sum);
    }
    float x = sum[0];
#pragma unroll
    for (int j = 1; j < 8; ++j) x = n == j ? sum[j] : x;
    if (n < 8) store_weight(w, b, tile, 8 * g + n, klen, there, x);
}

constexpr int kManyWaves = 8, kBlock = 256;        // queries whose buckets are in LDS together
struct ManyLds {
    int buck, table, sums, total;                  // after the queries' boxes
};
inline __host__ __device__ ManyLds many_lds(int nb, bool bias) {
    ManyLds l{};
    l.buck = bias ? kBlock * 16 : 0;
    l.table = l.buck + (bias ? kBlock * kBuckStride * 2 : 0);
    l.sums = l.table + (bias ? kManyWaves * ((nb * nb * 4 + 15) & ~15) : 0);
    l.total = l.sums + kManyWaves * kTile * 4;
    return l;
}

template <typename T, int DB, bool BIAS>
__global__ __launch_bounds__(kManyWaves * 64) void weigh_many_kernel(WeighArgs w) {
    using N = Num<T>;
    using Frag = typename N::Frag;
    extern __shared__ char smem[];
    const AttnArgs &a = w.a;
    const int tid = threadIdx.x, lane = tid & 63, n = lane & 15, g = lane >> 4;
    const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int64_t id = blockIdx.x;
    const int b = static_cast<int>(id / a.max_pages), tile = static_cast<int>(id % a.max_pages);
    const int klen = min(max(a.klen[b], 0), a.Nk), qlen = a.qlen ? min(max(a.qlen[b], 0), a.Nq) : a.Nq;
    const int page = tile * kTile < klen ? as_global<int32_t>(a.pages)[id] : -1;
    const bool there = page >= 0 && page < a.num_pages;
    if (!there || qlen == 0) {
        if (tid < kTile) store_weight(w, b, tile, tid, klen, there, 0.0f);
        return;
    }
    const ManyLds lds = many_lds(a.rule.nb, BIAS);
    const int nb2 = a.rule.nb * a.rule.nb;
    BoxGeo *geo = reinterpret_cast<BoxGeo *>(smem);
    uint16_t *buck = reinterpret_cast<uint16_t *>(smem + lds.buck);
    float *table = reinterpret_cast<float *>(smem + lds.table + wave * ((nb2 * 4 + 15) & ~15));
    float kx = 0.0f, ky = 0.0f;
    if (BIAS)
        box_centre(*(const REX_GLOBAL f32x4 *)(a.mbox + (static_cast<int64_t>(page) * kTile + (lane & 31)) * 4), kx, ky);
    uint32_t off[DB];
    code_offsets<DB>(a.D, n, g, off);

    float sum[8] = {};
    for (int q0 = 0; q0 < qlen; q0 += kBlock) {
        const int cols = min(qlen - q0, kBlock), tiles = (cols + 15) / 16;
        if (BIAS) {
            __syncthreads();
            if (tid < cols) geo[tid] = box_geo(box_load(a.qbox + b * a.qbox_sb + (q0 + tid) * a.qbox_sr));
            __syncthreads();
            for (int c = 2 * wave + (lane >> 5); c < 16 * tiles; c += 2 * kManyWaves)
                buck[c * kBuckStride + (lane & 31)] =
                    static_cast<uint16_t>(pair_bucket(geo[min(c, cols - 1)], kx, ky, a.rule));
            __syncthreads();
        }
        // a run of (head, 16 queries) for each wave
        const int all = a.H * tiles, per = (all + kManyWaves - 1) / kManyWaves;
        const int begin = min(wave * per, all), end = min(begin + per, all);
        Frag kf[2][DB];
        f32x4 ks[2];
        int head = -1;
        for (int i = begin; i < end; ++i) {
            const int h = i / tiles, at = (i - h * tiles) * 16;
            if (h != head) {
                if (head < 0 || h / a.group != head / a.group) {
                    KeyCodes<DB> codes;
                    load_codes<DB>(a, static_cast<int64_t>(page) * a.Hkv + h / a.group, off, g, codes);
                    widen_codes<T, DB>(codes, kf);
                    ks[0] = codes.s[0];
                    ks[1] = codes.s[1];
                }
                if (BIAS) {
                    gcptr<float> from = as_global<float>(a.bias + static_cast<int64_t>(h) * nb2);
                    asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");      // the last head's entries are read
                    for (int e = lane; e < nb2; e += 64) table[e] = from[e] <= kLowest ? -kInf : from[e];
                    asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
                }
                head = h;
            }
            const HeadRows qr = head_rows<T>(a.q, b, h, qlen, a.D);
            Frag q[1][DB];
            load_columns<T, DB, 1>(qr.at(q0 + at), qr.sr, n, g, a.D, q);
            const bool in = at + n < cols;
            const float lse = as_global<float>(w.lse)[(static_cast<int64_t>(b) * a.H + h) * a.Nq + q0 + (in ? at + n : 0)];
            f32x4 bias[2] = {};
            if (BIAS)
                table_gather(*reinterpret_cast<const u32x4 *>(buck + (at + n) * kBuckStride + 8 * g),
                             reinterpret_cast<const char *>(table), bias);
            add_weights<T, DB>(kf, ks, q[0], bias, a.scale, lse, in && fabsf(lse) < kInf, sum);
        }
    }
    sum_columns(sum);
    float x = sum[0];
#pragma unroll
    for (int j = 1; j < 8; ++j) x = n == j ? sum[j] : x;
    float *sums = reinterpret_cast<float *>(smem + lds.sums);
    if (n < 8) sums[wave * kTile + 8 * g + n] = x;
    __syncthreads();
    if (tid >= kTile) return;
    x = sums[tid];
#pragma unroll
    for (int i = 1; i < kManyWaves; ++i) x += sums[i * kTile + tid];
    store_weight(w, b, tile, tid, klen, there, x);
}

template <typename T, int DB> void run(const WeighArgs &w, hipStream_t s) {
    const int64_t pages = static_cast<int64_t>(w.a.B) * w.a.max_pages;
    if (w.a.Nq <= kFewQueries) {
        const uint32_t grid = static_cast<uint32_t>((pages + kFewWaves - 1) / kFewWaves);
        if (w.a.bias) weigh_few_kernel<T, DB, true><<<grid, kFewWaves * 64, 0, s>>>(w);
        else weigh_few_kernel<T, DB, false><<<grid, kFewWaves * 64, 0, s>>>(w);
        return;
    }
    const uint32_t grid = static_cast<uint32_t>(pages), lds = many_lds(w.a.rule.nb, w.a.bias != nullptr).total;
    if (w.a.bias) weigh_many_kernel<T, DB, true><<<grid, kManyWaves * 64, lds, s>>>(w);
    else weigh_many_kernel<T, DB, false><<<grid, kManyWaves * 64, lds, s>>>(w);
}
template <typename T> void run_sized(const WeighArgs &w, hipStream_t s) {
    if (w.a.D <= 32) run<T, 1>(w, s);
    else if (w.a.D <= 64) run<T, 2>(w, s);
    else run<T, 4>(w, s);
}

}  // namespace

hipError_t launch_weigh(const WeighArgs &w, int dtype, hipStream_t s) {
    if (dtype == kF32) run_sized<float>(w, s);
    else run_sized<uint16_t>(w, s);
    return hipGetLastError();
}

}  // namespace rex
