// weigh.hip -- the attention that each remembered box has received (box_memory_weigh).
//
// Sums over keys are not needed, the log sum is given, and so nothing but half of the memory is
// read: codes and scales of the keys, and the boxes.
//
// One to four rows that share a key head's keys (queries times the heads of a group): a lane has a box,
// half a wave a key head, and products are sums of its lane: of sixteen columns of a matrix product
// fifteen would be empty, and what is done with its results as well.  64 streams of 8192 boxes in 8 heads
// of 32: one row 43 us with nothing in the caches (143 MB at 3.4 TB/s), 37 with two sets of inputs in turn; and
// where the same call is repeated, as in all that follows, 28, as columns 91; four 53 and 98; 16 streams in 16
// heads of 64: 45 and 56, 62 and 62.
//
// More: the logits are made as in the recall (attn_fwd.hpp), keys the rows of the products and queries
// their columns, so a lane has eight keys of one query, and adds their weights up over heads and
// queries in its registers; the sixteen lanes of a row meet at the end, once for a page.  Up to 16 queries
// a wave takes a page and all of its heads, several heads' codes on their way at once: 16 rows of those 64
// streams 107 us.  Beyond, a workgroup takes a page, its waves share heads and queries out, and the buckets
// of 256 queries against the page's boxes are computed once for all heads into LDS: 17 rows 123 us (155 the
// other way), 128 249 (617); 300 rows against 6000 boxes in 16 heads of 64, 31, of binary32 queries 64, whose
// products take sixteen times as many matrix cycles: vector instructions bound the former, half of the time of
// the 188 CUs that have a page.
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

// exp2(min(d, 0)) of a logit less its row's log sum, in units of log 2, and 0 where d is NaN (the median of
// three is their least where one of them is NaN; with -inf for the lowest the compiler would leave it out): a
// NaN logit adds nothing, nor does any logit, NaN and +inf among them, less the +inf of a row that is none.
__device__ __forceinline__ float weight_of(float d) {
    return __builtin_amdgcn_exp2f(__builtin_amdgcn_fmed3f(d, 0.0f, -3e38f));
}

// Adds a column's weights of eight keys, in units of log 2: ks the codes' scales times that of the
// logits, bias by key, lse as row_reference has it.
template <typename T, int DB>
__device__ __forceinline__ void add_weights(const typename Num<T>::Frag (&kf)[2][DB], const f32x4 (&ks)[2],
                                            const typename Num<T>::Frag (&q)[DB], const f32x4 (&bias)[2], float lse,
                                            float (&sum)[8]) {
    f32x4 x[2] = {};
#pragma unroll
    for (int t = 0; t < 2; ++t)
#pragma unroll
        for (int k = 0; k < DB; ++k) x[t] = Num<T>::mma(kf[t][k], q[k], x[t]);
#pragma unroll
    for (int j = 0; j < 8; ++j)
        sum[j] += weight_of(fmaf(x[j >> 2][j & 3], ks[j >> 2][j & 3], bias[j >> 2][j & 3]) - lse);
}
// A row's log sum in units of log 2, +inf where the row adds nothing.
__device__ __forceinline__ float row_reference(float lse, bool in) {
    return in && fabsf(lse) < kInf ? lse * kLog2e : kInf;
}
// The scale of a lane's eight keys, of their logits in units of log 2.
__device__ __forceinline__ void logit_scales(f32x4 (&s)[2], float scale) {
    s[0] *= scale;
    s[1] *= scale;
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
                    lse[i] = row_reference(lse[i], n < qlen && first + i < a.Hkv);
                    bias[i][0] = bias[i][1] = f32x4{};
                    if (BIAS && n < qlen) {
                        const float *table = a.bias + static_cast<int64_t>(h) * a.rule.nb * a.rule.nb;
#pragma unroll
                        for (int j = 0; j < 8; ++j) bias[i][j >> 2][j & 3] = wide_entry(table, at[j]) * kLog2e;
                    }
                }
#pragma unroll
                for (int i = 0; i < kHeads; ++i) {
                    Frag kf[2][DB];
                    widen_codes<T, DB>(codes[i], kf);
                    f32x4 ks[2] = {codes[i].s[0], codes[i].s[1]};
                    logit_scales(ks, a.scale * kLog2e);
                    add_weights<T, DB>(kf, ks, q[i], bias[i], lse[i], sum);
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

// A lane for each box of a page and half of its key heads; COMBOS rows that share a key head's keys
// (`rows` queries of each of a group's heads), whose queries lie in LDS as binary32, key head after key
// head.
constexpr int kLaneWaves = 4, kLanePages = 2;      // pages of a wave, one after the other
constexpr int kLaneBytes = 32 << 10;               // of LDS, for queries

template <typename T, int COMBOS, bool BIAS>
__global__ __launch_bounds__(kLaneWaves * 64) void weigh_lane_kernel(WeighArgs w, int blocks) {
    extern __shared__ char smem[];
    const AttnArgs &a = w.a;
    float *queries = reinterpret_cast<float *>(smem);          // [Hkv][D / 4][COMBOS][4]
    float *refs = queries + a.Hkv * a.D * COMBOS;              // [Hkv][COMBOS]
    const int tid = threadIdx.x, lane = tid & 63, r = lane & 31, half = lane >> 5;
    const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int b = blockIdx.x / blocks, block = blockIdx.x % blocks;
    const int klen = min(max(a.klen[b], 0), a.Nk), qlen = a.qlen ? min(max(a.qlen[b], 0), a.Nq) : a.Nq;
    const int nq = a.Nq, nb2 = a.rule.nb * a.rule.nb;
    if (block * kLaneWaves * kLanePages * kTile < klen && qlen > 0) {
        // combo c: head c / nq of the group, query c % nq
        for (int i = tid; i < a.Hkv * COMBOS; i += kLaneWaves * 64) {
            const int kh = i / COMBOS, c = i % COMBOS, of = c / nq, row = c % nq;
            const bool in = of < a.group && row < qlen;
            const float lse = in ? as_global<float>(w.lse)[(static_cast<int64_t>(b) * a.H + kh * a.group + of) * nq + row] : kInf;
            refs[i] = row_reference(lse, in);
        }
        for (int i = tid; i < a.Hkv * a.D * COMBOS; i += kLaneWaves * 64) {
            const int e = i & 3, c = (i >> 2) % COMBOS, rest = (i >> 2) / COMBOS, kh = rest / (a.D / 4);
            const int ch = rest % (a.D / 4) * 4 + e, of = c / nq, row = c % nq, h = kh * a.group + of;
            float x = 0.0f;
            if (of < a.group && row < qlen)
                x = load_f32<T>(as_global<T>(static_cast<const char *>(a.q.p) + b * a.q.sb + static_cast<int64_t>(row) * a.q.sr +
                                             static_cast<int64_t>(h) * a.q.sh) + ch);
            queries[i] = x;
        }
    }
    __syncthreads();
    for (int i = 0; i < kLanePages; ++i) {
        const int tile = (block * kLanePages + i) * kLaneWaves + wave;
        if (tile >= a.max_pages) return;
        const int page = tile * kTile < klen ? as_global<int32_t>(a.pages)[static_cast<int64_t>(b) * a.max_pages + tile] : -1;
        const bool there = page >= 0 && page < a.num_pages;
        float sum = 0.0f;
        if (there && qlen > 0) {
            uint32_t at[COMBOS];                    // a combo's entry in its head's table
            if (BIAS) {
                float kx, ky;
                box_centre(*(const REX_GLOBAL f32x4 *)(a.mbox + (static_cast<int64_t>(page) * kTile + r) * 4), kx, ky);
#pragma unroll
                for (int c = 0; c < COMBOS; ++c) {
                    const BoxGeo geo = box_geo(box_load(a.qbox + b * a.qbox_sb + min(c % nq, qlen - 1) * a.qbox_sr));
                    at[c] = pair_bucket(geo, kx, ky, a.rule) / 4 + min(c / nq, a.group - 1) * nb2;
                }
            }
            const int64_t head0 = static_cast<int64_t>(page) * a.Hkv;
#pragma unroll 2
            for (int kh = half; kh < a.Hkv; kh += 2) {
                const float scale = as_global<float>(a.mks)[(head0 + kh) * kTile + r] * (a.scale * kLog2e);
                const int8_t *row = a.mk + ((head0 + kh) * kTile + r) * a.D;
                const f32x4 *q = reinterpret_cast<const f32x4 *>(queries) + kh * (a.D / 4) * COMBOS;
                float dot[COMBOS] = {};
                for (int c0 = 0; c0 < a.D; c0 += 32) {         // (D is a multiple of 8)
                    u32x2 codes[4] = {};
#pragma unroll
                    for (int k = 0; k < 4; ++k)
                        if (c0 + 8 * k < a.D) codes[k] = *(const REX_GLOBAL u32x2 *)(row + c0 + 8 * k);
#pragma unroll
                    for (int k = 0; k < 8; ++k) {
                        if (c0 + 4 * k >= a.D) break;
                        const uint32_t x = codes[k >> 1][k & 1];
#pragma unroll
                        for (int c = 0; c < COMBOS; ++c) {
                            const f32x4 y = q[(c0 / 4 + k) * COMBOS + c];
#pragma unroll
                            for (int e = 0; e < 4; ++e)
                                dot[c] = fmaf(static_cast<float>(static_cast<int8_t>(x >> (8 * e))), y[e], dot[c]);
                        }
                    }
                }
#pragma unroll
                for (int c = 0; c < COMBOS; ++c) {
                    float bias = 0.0f;
                    if (BIAS) bias = wide_entry(a.bias + static_cast<int64_t>(kh) * a.group * nb2, 4 * at[c]) * kLog2e;
                    sum += weight_of(fmaf(dot[c], scale, bias) - refs[kh * COMBOS + c]);
                }
            }
            sum += __shfl_xor(sum, 32);
        }
        if (half == 0) store_weight(w, b, tile, r, klen, there, sum);
    }
}
// Rows that share keys, rounded up; 0: too many, or too much LDS.
int lane_combos(const AttnArgs &a) {
    const int64_t rows = static_cast<int64_t>(a.Nq) * a.group;
    const int c = rows <= 1 ? 1 : rows <= 2 ? 2 : rows <= 4 ? 4 : 0;
    return c * a.Hkv * (a.D + 1) * 4 <= kLaneBytes ? c : 0;
}

constexpr int kBlock = 256;        // queries whose buckets are in LDS together
struct ManyLds {
    int buck, table, sums, total;                  // after the queries' boxes
};
inline __host__ __device__ ManyLds many_lds(int nb, bool bias, int waves) {
    ManyLds l{};
    l.buck = bias ? kBlock * 16 : 0;
    l.table = l.buck + (bias ? kBlock * kBuckStride * 2 : 0);
    l.sums = l.table + (bias ? waves * ((nb * nb * 4 + 15) & ~15) : 0);
    l.total = l.sums + waves * kTile * 4;
    return l;
}

template <typename T, int DB, bool BIAS, int WAVES>
__global__ __launch_bounds__(WAVES * 64) void weigh_many_kernel(WeighArgs w) {
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
    const ManyLds lds = many_lds(a.rule.nb, BIAS, WAVES);
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
            for (int c = 2 * wave + (lane >> 5); c < 16 * tiles; c += 2 * WAVES)
                buck[c * kBuckStride + (lane & 31)] =
                    static_cast<uint16_t>(pair_bucket(geo[min(c, cols - 1)], kx, ky, a.rule));
            __syncthreads();
        }
        // a run of (head, 16 queries) for each wave, the next one's queries on their way
        const int all = a.H * tiles, per = (all + WAVES - 1) / WAVES;
        const int begin = min(wave * per, all), end = min(begin + per, all);
        Frag kf[2][DB], next[1][DB];
        f32x4 ks[2];
        float next_lse = 0.0f;
        const auto load_rows = [&](int h, int at) {
            const HeadRows qr = head_rows<T>(a.q, b, h, qlen, a.D);
            load_columns<T, DB, 1>(qr.at(q0 + at), qr.sr, n, g, a.D, next);
            next_lse = as_global<float>(w.lse)[(static_cast<int64_t>(b) * a.H + h) * a.Nq + q0 + min(at + n, cols - 1)];
        };
        int h = begin / tiles, at = begin % tiles * 16, head = -1;
        if (begin < end) load_rows(h, at);
        for (int i = begin; i < end; ++i) {
            if (h != head) {
                if (head < 0 || h / a.group != head / a.group) {
                    KeyCodes<DB> codes;
                    load_codes<DB>(a, static_cast<int64_t>(page) * a.Hkv + h / a.group, off, g, codes);
                    widen_codes<T, DB>(codes, kf);
                    ks[0] = codes.s[0];
                    ks[1] = codes.s[1];
                    logit_scales(ks, a.scale * kLog2e);
                }
                if (BIAS) {
                    gcptr<float> from = as_global<float>(a.bias + static_cast<int64_t>(h) * nb2);
                    asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");      // the last head's entries are read
                    for (int e = lane; e < nb2; e += 64) table[e] = from[e] <= kLowest ? -kInf : from[e] * kLog2e;
                    asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
                }
                head = h;
            }
            Frag q[DB];
#pragma unroll
            for (int k = 0; k < DB; ++k) q[k] = next[0][k];
            const float lse = row_reference(next_lse, at + n < cols);
            const int here = at;
            at += 16;
            if (at >= 16 * tiles) {
                at = 0;
                ++h;
            }
            if (i + 1 < end) load_rows(h, at);
            f32x4 bias[2] = {};
            if (BIAS)
                table_gather(*reinterpret_cast<const u32x4 *>(buck + (here + n) * kBuckStride + 8 * g),
                             reinterpret_cast<const char *>(table), bias);
            add_weights<T, DB>(kf, ks, q, bias, lse, sum);
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
    for (int i = 1; i < WAVES; ++i) x += sums[i * kTile + tid];
    store_weight(w, b, tile, tid, klen, there, x);
}

template <typename T, int COMBOS> void run_lane(const WeighArgs &w, hipStream_t s) {
    const int blocks = (w.a.max_pages + kLaneWaves * kLanePages - 1) / (kLaneWaves * kLanePages);
    const uint32_t grid = static_cast<uint32_t>(w.a.B) * blocks, lds = COMBOS * w.a.Hkv * (w.a.D + 1) * 4;
    if (w.a.bias) weigh_lane_kernel<T, COMBOS, true><<<grid, kLaneWaves * 64, lds, s>>>(w, blocks);
    else weigh_lane_kernel<T, COMBOS, false><<<grid, kLaneWaves * 64, lds, s>>>(w, blocks);
}

template <typename T, int DB, int WAVES> void run_many(const WeighArgs &w, hipStream_t s) {
    const uint32_t grid = static_cast<uint32_t>(w.a.B) * w.a.max_pages;
    const uint32_t lds = many_lds(w.a.rule.nb, w.a.bias != nullptr, WAVES).total;
    if (w.a.bias) weigh_many_kernel<T, DB, true, WAVES><<<grid, WAVES * 64, lds, s>>>(w);
    else weigh_many_kernel<T, DB, false, WAVES><<<grid, WAVES * 64, lds, s>>>(w);
}

template <typename T, int DB> void run(const WeighArgs &w, hipStream_t s) {
    const int64_t pages = static_cast<int64_t>(w.a.B) * w.a.max_pages;
    switch (lane_combos(w.a)) {
    case 1: return run_lane<T, 1>(w, s);
    case 2: return run_lane<T, 2>(w, s);
    case 4: return run_lane<T, 4>(w, s);
    }
    if (w.a.Nq <= kFewQueries) {
        const uint32_t grid = static_cast<uint32_t>((pages + kFewWaves - 1) / kFewWaves);
        if (w.a.bias) weigh_few_kernel<T, DB, true><<<grid, kFewWaves * 64, 0, s>>>(w);
        else weigh_few_kernel<T, DB, false><<<grid, kFewWaves * 64, 0, s>>>(w);
        return;
    }
    // Four waves a page where pages fill the GPU several times over, sixteen where they do not (eight for
    // wide binary32 heads, whose operands fill more registers).  16 streams of 8192 boxes in 16 heads of 64
    // against 32 rows: 74 us with 4 waves, 86 with 8, 126 with 16; one of 6000 against 300: 50, 34 and 33.
    constexpr int kWide = DB == 4 && sizeof(T) == 4 ? 8 : 16;
    if (pages >= 512) run_many<T, DB, 4>(w, s);
    else run_many<T, DB, kWide>(w, s);
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
