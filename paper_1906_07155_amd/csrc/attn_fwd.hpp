// attn_fwd.hpp -- the forward of the attention among boxes, over dense keys (box_attn_fwd)
// or over the 8-bit memory (box_memory_attn_fwd).
//
// One workgroup of eight waves owns 16 * NS query rows of one image and `hp` heads; wave w
// takes head w % hp and every (8 / hp)-th tile of 32 keys.  Each wave makes one pass over
// its keys with the running maximum and sum of the softmax; queries are the columns of every
// product, so maximum, sum and rescaling are per lane, and the weights go from one product
// into the next without leaving their lane (attn.hpp).  Where the waves of a head share the
// keys, their sums meet in LDS at the end; where that still leaves the GPU empty (few rows, a
// long memory) the keys are split over workgroups as well and attn_combine joins them.
//
// The bucket of a pair is the same for all heads, and costs more than one head's
// share of the products: the workgroup computes each tile's buckets once, a step ahead,
// into LDS (16 bits a pair: the byte offset into a head's table, which is in LDS too).
//
// Measured, bf16: 100 boxes in 8 heads of 32 channels 9.7 us (a launch and four dependent
// steps); 1000 in 16 heads of 64 29.5 us; 16 images of 600 to 1000 of those and one of none 210 us:
// some 40 GFLOP of products, 60 with the second part of the weights, that take 53 us at the rate of a
// large product; vector instructions (bias, exponent, running maximum, parts of the weights) take half
// of the CUs' time.  1000 boxes in 8 heads of 128: 43 us.  64 single queries against 1000 keys each in
// 8 heads of 32: 23.5 us, in binary32 33.
// The memory, 300 boxes against 6000 in 16 heads of 64: 56 us, in binary32 111; 64 single queries
// against up to 8192 in 8 heads of 32: 83 us, 3.3 TB/s, in binary32 126.
#pragma once

#include "attn.hpp"

namespace rex {

// Exponents whose rounding is no longer far below 1: beyond, they are taken from the maximum itself.
constexpr float kFarExponent = 1024.0f;

// What is in LDS, in bytes from its start.
struct FwdLds {
    int bias, geo, buck, tile, ref, near, acc, total;
};
// Steps whose buckets are computed between two barriers.
inline __host__ __device__ int fwd_ahead(int parts) { return parts >= 2 ? 1 : 2; }
inline __host__ __device__ FwdLds fwd_lds(int cols, int dp, int hp, int parts, int nb, bool bias, int tiles) {
    FwdLds l{};
    int at = 0;
    l.bias = at;
    if (bias) at += (hp * nb * nb * 4 + 15) & ~15;
    l.geo = at;
    if (bias) at += cols * 16;
    l.buck = at;
    if (bias) at += 2 * fwd_ahead(parts) * parts * cols * kBuckStride * 2;
    l.tile = at;
    at += kAttnWaves * tiles * kTile * dp * 2;        // each wave's tiles of bf16 rows
    const int loop = at;
    at = 0;                       // the end: the loop's tables are no longer needed
    l.ref = at;
    if (parts > 1) at += hp * parts * cols * static_cast<int>(sizeof(SumRef));
    l.near = at;
    if (parts > 1) at += hp * parts * cols * 4;
    l.acc = at;
    if (parts > 1) at += hp * parts * cols * (dp + 4) * 4;
    l.total = at > loop ? at : loop;
    return l;
}

// Tiles of bf16 rows that a wave keeps in LDS, keys and values, or values alone for
// heads of more than 64 channels.  (Two of each, the next on its way for a whole step, leave room
// for one workgroup on a CU instead of two: 1000 queries and keys in 16 heads of 64 channels, weights in
// one part, take 27.2 us then, 26.2 as it is.)
template <typename T, int DB, bool PAGED>
constexpr int fwd_tiles() { return PAGED || sizeof(T) == 4 ? 0 : DB <= 2 ? 2 : 1; }

// The sums of a row's parts are joined relative to the part whose exponent is the largest.  Both
// differences are exact wherever they are small enough to matter; a part without a key has none.
__device__ __forceinline__ float ref_gap(const SumRef &p, const SumRef &to) {
    const float gap = (p.offset - to.offset) * kLog2e + static_cast<float>(p.rest - to.rest);
    return p.rest == -static_cast<double>(kInf) ? -kInf : gap;
}
__device__ __forceinline__ void reach(SumRef &to, const SumRef &p) {
    if (to.rest == -static_cast<double>(kInf) || ref_gap(p, to) > 0.0f) to = p;
}
__device__ __forceinline__ SumRef load_ref(const SumRef *p) {
    const f32x4 x = *(const REX_GLOBAL f32x4 *)(p);
    return __builtin_bit_cast(SumRef, x);
}
__device__ __forceinline__ float row_lse(const SumRef &r) {
    if (r.sum == 0.0f) return -kInf;
    return static_cast<float>((r.rest + log2f(r.sum)) * 0.69314718055994530942 + r.offset);
}

template <typename T, int DB, int NS, bool BIAS, bool PAGED, int TERMS>
__global__ __launch_bounds__(kAttnWaves * 64, 2) void attn_fwd_kernel(AttnArgs a) {
    using N = Num<T>;
    using Frag = typename N::Frag;
    using Pair = typename N::Pair;
    constexpr int kCols = 16 * NS, kDP = 32 * DB;
    constexpr bool kLds = !PAGED && sizeof(T) == 2, kNatural = PAGED || kLds;
    constexpr bool kBoth = fwd_tiles<T, DB, PAGED>() == 2;
    extern __shared__ char smem[];
    const int id = xcd_order(blockIdx.x, a.nwg, a.per);
    if (id >= a.nwg) return;
    const int tid = threadIdx.x, lane = tid & 63, n = lane & 15, g = lane >> 4;
    const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int hp = a.hp, parts = a.parts, hw = wave & (hp - 1), kw = wave / hp;
    int rest = id;
    const int tile_q = rest % a.tiles;
    rest /= a.tiles;
    const int split = rest % a.nsplit;
    rest /= a.nsplit;
    const int hgroups = a.H / hp;
    const int h0 = (rest % hgroups) * hp, b = rest / hgroups;
    const int h = h0 + hw, kh = h / a.group;
    const int ahead = fwd_ahead(parts);
    const FwdLds lds = fwd_lds(kCols, kDP, hp, parts, a.rule.nb, BIAS, fwd_tiles<T, DB, PAGED>());

    const int qlen = a.qlen ? min(max(a.qlen[b], 0), a.Nq) : a.Nq;
    const int klen = a.klen ? min(max(a.klen[b], 0), a.Nk) : a.Nk;
    const int q0 = tile_q * kCols;
    const int all = (klen + kTile - 1) / kTile;
    const int per = (all + a.nsplit - 1) / a.nsplit;
    const int t0 = min(split * per, all), t1 = q0 < qlen ? min(t0 + per, all) : t0;

    const int cols = min(max(qlen - q0, 0), kCols);       // columns that hold a query
    BoxGeo *geo = reinterpret_cast<BoxGeo *>(smem + lds.geo);
    uint16_t *buck = reinterpret_cast<uint16_t *>(smem + lds.buck);
    const int nb2 = a.rule.nb * a.rule.nb;
    if (BIAS) {
        float *t = reinterpret_cast<float *>(smem + lds.bias);
        gcptr<float> src = as_global<float>(a.bias + static_cast<int64_t>(h0) * nb2);
        for (int i = tid; i < hp * nb2; i += kAttnWaves * 64) t[i] = table_entry(src[i], a.scale);
        if (tid < cols) geo[tid] = box_geo(box_load(a.qbox + b * a.qbox_sb + (q0 + tid) * a.qbox_sr));
        // columns without a query: bucket 0 of whatever they hold
        if (cols < kCols)
            for (int i = tid; i < 2 * ahead * parts * kCols * kBuckStride / 2; i += kAttnWaves * 64)
                reinterpret_cast<uint32_t *>(buck)[i] = 0u;
    }

    // the queries: column n of NS tiles; rows that are padding are zeros
    Frag q[NS][DB];
    {
        const HeadRows qr = head_rows<T>(a.q, b, h, qlen, a.D);
        load_columns<T, DB, NS>(qr.at(min(q0, max(qlen - 1, 0))), qr.sr, n, g, a.D, q);
    }

    // One tile's keys and values, its page and the lane's mask byte, read one step ahead.
    const HeadRows kr = head_rows<T>(a.k, b, kh, PAGED ? 0 : klen, a.D);
    const HeadRows vr = head_rows<T>(a.v, b, kh, PAGED ? 0 : klen, a.D);
    const TileOffsets<T, DB> koff(kr.sr, n, g, a.D), voff(vr.sr, n, g, a.D);
    const LdsTile<DB> rows(smem + lds.tile + wave * fwd_tiles<T, DB, PAGED>() * LdsTile<DB>::kBytes, lane);
    const typename LdsTile<DB>::Loads kload(kr.sr, lane, a.D), vload(vr.sr, lane, a.D);
    // the same inside a page of the memory; its values' channels past D are past its end
    uint32_t kcode[DB];
    const uint32_t vcode = n * kTile + 8 * g;
#pragma unroll
    for (int k = 0; k < DB; ++k)
        kcode[k] = 32 * k + 8 * g < a.D ? (8 * (n >> 2) + (n & 3)) * a.D + 32 * k + 8 * g : kBufOOB;
    struct {
        Frag f[2][DB];                                   // keys
        Pair p[DB][8];                                   // values (binary32)
        u32x2 kc[PAGED ? 2 : 1][PAGED ? DB : 1];         // their codes and scales in the memory
        u32x2 vc[PAGED ? 2 * DB : 1];
        f32x4 ks[2], vs[2];
        int64_t ph;
        bool on;
    } next;
    // The pages of this wave's next 64 tiles are read at once, one by each lane.
    struct Pages {
        int v;
        __device__ __forceinline__ int get(const AttnArgs &a, int b, int first, int parts, int step, int end) {
            if ((step & 63) == 0) {
                const int at = first + (step + static_cast<int>(threadIdx.x & 63)) * parts;
                v = at < end ? as_global<int32_t>(a.pages)[static_cast<int64_t>(b) * a.max_pages + at] : -1;
            }
            const int p = __builtin_amdgcn_readlane(v, step & 63);
            return p >= 0 && p < a.num_pages ? p : -1;
        }
    } kpages, bpages;
    kpages.v = bpages.v = -1;
    int kstep = 0;                                       // load_keys takes this wave's tiles in order
    auto load_keys = [&](int tile) {
        const int key = tile * kTile + (lane & 31);
        next.on = key < klen;
        if constexpr (PAGED) {
            const int page = kpages.get(a, b, t0 + kw, parts, kstep++, t1);
            next.on = next.on && page >= 0;
            next.ph = static_cast<int64_t>(max(page, 0)) * a.Hkv + kh;
            const auto r = make_rsrc(a.mk + next.ph * kTile * a.D, kTile * a.D);
#pragma unroll
            for (int t = 0; t < 2; ++t) {
                next.ks[t] = *(const REX_GLOBAL f32x4 *)(a.mks + next.ph * kTile + 8 * g + 4 * t);
#pragma unroll
                for (int k = 0; k < DB; ++k)
                    next.kc[t][k] = __builtin_amdgcn_raw_buffer_load_b64(r, kcode[k], 4 * t * a.D, 0);
            }
        } else {
            if (a.kmask)
                next.on = next.on && as_global<uint8_t>(a.kmask)[static_cast<int64_t>(b) * a.Nk + min(key, a.Nk - 1)] != 0;
            const auto r = kr.at(tile * kTile);
            const bool inside = tile * kTile + kTile <= klen;
            if constexpr (kBoth) rows.fill(r, inside, kload);
            else koff.frags(r, inside, next.f);
        }
    };
    auto load_values = [&](int tile) {                   // after load_keys of the same tile
        if constexpr (PAGED) {
            const auto r = make_rsrc(a.mv + next.ph * kTile * a.D, kTile * a.D);
#pragma unroll
            for (int t = 0; t < 2; ++t)
                next.vs[t] = *(const REX_GLOBAL f32x4 *)(a.mvs + next.ph * kTile + 8 * g + 4 * t);
#pragma unroll
            for (int u = 0; u < 2 * DB; ++u)
                next.vc[u] = __builtin_amdgcn_raw_buffer_load_b64(r, vcode + 16 * kTile * u, 0, 0);
        } else if constexpr (kLds) {
            rows.fill(vr.at(tile * kTile), tile * kTile + kTile <= klen, vload, kBoth ? 1 : 0);
        } else {
            voff.pairs(vr.at(tile * kTile), tile * kTile + kTile <= klen, next.p);
        }
    };
    // Buckets of the chunk's tiles against the workgroup's queries, by the waves that read them;
    // the boxes are read a chunk before.
    f32x4 kb[2];
    auto load_boxes = [&](int chunk) {
        const int r = lane & 31;
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            const int step = chunk * ahead + i, tile = t0 + step * parts + kw;
            if (i >= ahead || tile >= t1) return;
            if constexpr (PAGED)
                kb[i] = *(const REX_GLOBAL f32x4 *)(
                    a.mbox + (static_cast<int64_t>(max(bpages.get(a, b, t0 + kw, parts, step, t1), 0)) * kTile + r) * 4);
            else kb[i] = box_load(a.kbox + b * a.kbox_sb + min(tile * kTile + r, a.Nk - 1) * a.kbox_sr);
        }
    };
    auto fill_buckets = [&](int chunk) {
        const int r = lane & 31;
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            if (i >= ahead || t0 + (chunk * ahead + i) * parts + kw >= t1) return;
            float kx, ky;
            box_centre(kb[i], kx, ky);
            uint16_t *dst = buck + (((chunk & 1) * ahead + i) * parts + kw) * kCols * kBuckStride + r;
#pragma unroll 2
            for (int c = hw * 2 + (lane >> 5); c < cols; c += 2 * hp)
                dst[c * kBuckStride] = static_cast<uint16_t>(pair_bucket(geo[c], kx, ky, a.rule));
        }
    };

    const float sl2 = a.scale * kLog2e;
    const char *tab = smem + lds.bias + hw * nb2 * 4;
    f32x4 o[NS][2 * DB] = {};      // 16-channel tiles 2k, 2k + 1: even and odd channels
    // The running maximum, in units of the products; what exponents are taken from (m in units
    // of log 2, 0 while there is no key); the sum.  Where logits are so large that m in units of
    // log 2 would be off by a part of 1 (`far`), m is taken off the logits first and ref is 0.  With
    // a wide table m and the products' sums are relative to the row's largest entry so far.
    float m[NS], ref[NS], l[NS], offset[NS];
    bool far = false, wide = false;     // (wide: wide_table)
    const float slack = 8.0f / sl2, per_scale = 1.0f / a.scale;
#pragma unroll
    for (int s = 0; s < NS; ++s) {
        m[s] = -kInf;
        ref[s] = l[s] = offset[s] = 0.0f;
    }
    const int steps = (t1 - t0 + parts - 1) / parts, chunks = (steps + ahead - 1) / ahead;
    if (t0 + kw < t1) {
        load_keys(t0 + kw);
        load_values(t0 + kw);
    }
    if (BIAS) {
        load_boxes(0);
        __syncthreads();
        wide = far = wide_table(tab, nb2, a.scale, lane);
#pragma unroll
        for (int s = 0; s < NS; ++s) offset[s] = wide ? -kInf : 0.0f;
        fill_buckets(0);
        load_boxes(1);
    }

    for (int chunk = 0; chunk < chunks; ++chunk) {
        if (BIAS) {
            __syncthreads();
            if (chunk + 1 < chunks) fill_buckets(chunk + 1);
            load_boxes(chunk + 2);
        }
        for (int i = 0; i < ahead; ++i) {
            const int tile = t0 + (chunk * ahead + i) * parts + kw;
            if (tile >= t1) break;
            const uint32_t vis = static_cast<uint32_t>(__ballot(next.on));   // bit r: key r is visible
            const bool more = tile + parts < t1;
            if constexpr (kLds) rows.arrived();
            Frag vf[2 * DB];
            if constexpr (kLds) {
#pragma unroll
                for (int u = 0; u < 2 * DB; ++u) vf[u] = rows.channels(u, kBoth ? 1 : 0);
            }
            // what a logit starts with: its bias, or nothing
            f32x4 x[NS][2];
            const uint16_t *bk = buck + ((((chunk & 1) * ahead + i) * parts + kw) * kCols + n) * kBuckStride + 8 * g;
#pragma unroll
            for (int s = 0; s < NS; ++s) {
                x[s][0] = x[s][1] = f32x4{};
                if (BIAS) table_gather(*reinterpret_cast<const u32x4 *>(bk + 16 * s * kBuckStride), tab, x[s]);
            }
            if (BIAS && __builtin_expect(wide, 0)) {
#pragma unroll
                for (int s = 0; s < NS; ++s) {
                    wide_gather(*reinterpret_cast<const u32x4 *>(bk + 16 * s * kBuckStride),
                                a.bias + static_cast<int64_t>(h) * nb2, x[s]);
                    float top = -kInf;
#pragma unroll
                    for (int j = 0; j < 8; ++j) top = vis >> (8 * g + j) & 1u ? fmaxf(top, x[s][j >> 2][j & 3]) : top;
                    top = max_over_rows(top);
                    if (top > offset[s]) {       // m is where it was, as seen from the new offset
                        m[s] -= (top - offset[s]) * per_scale;
                        offset[s] = top;
                    }
                    const float from = offset[s] == -kInf ? 0.0f : offset[s];
#pragma unroll
                    for (int j = 0; j < 8; ++j) x[s][j >> 2][j & 3] = (x[s][j >> 2][j & 3] - from) * per_scale;
                }
            }
            // column = query n, rows = keys 8g + 4t + e
#pragma unroll
            for (int t = 0; t < 2; ++t) {
                Frag kf[DB];
#pragma unroll
                for (int k = 0; k < DB; ++k) {
                    if constexpr (PAGED) {
                        N::widen(kf[k], 0, next.kc[t][k][0]);
                        N::widen(kf[k], 4, next.kc[t][k][1]);
                    } else if constexpr (kBoth) {
                        kf[k] = rows.rows(t, k);
                    } else {
                        kf[k] = next.f[t][k];
                    }
                }
#pragma unroll
                for (int s = 0; s < NS; ++s) {
                    if constexpr (PAGED) {
                        f32x4 acc = {};
#pragma unroll
                        for (int k = 0; k < DB; ++k) acc = N::mma(kf[k], q[s][k], acc);
#pragma unroll
                        for (int e = 0; e < 4; ++e) x[s][t][e] = fmaf(acc[e], next.ks[t][e], x[s][t][e]);
                    } else {
#pragma unroll
                        for (int k = 0; k < DB; ++k) x[s][t] = N::mma(kf[k], q[s][k], x[s][t]);
                    }
                }
            }
            f32x4 vs[2];
            if constexpr (PAGED) {
#pragma unroll
                for (int t = 0; t < 2; ++t) vs[t] = next.vs[t];
#pragma unroll
                for (int u = 0; u < 2 * DB; ++u) {
                    N::widen(vf[u], 0, next.vc[u][0]);
                    N::widen(vf[u], 4, next.vc[u][1]);
                }
            } else if constexpr (!kLds) {
#pragma unroll
                for (int k = 0; k < DB; ++k) N::split(next.p[k], vf[2 * k], vf[2 * k + 1]);
            }
            if (vis != 0xffffffffu) {
                const uint32_t mine = vis >> (8 * g);
#pragma unroll
                for (int j = 0; j < 8; ++j) {
                    const bool on = mine >> j & 1u;
#pragma unroll
                    for (int s = 0; s < NS; ++s) x[s][j >> 2][j & 3] = on ? x[s][j >> 2][j & 3] : -kInf;
                    if constexpr (PAGED) vs[j >> 2][j & 3] = on ? vs[j >> 2][j & 3] : 0.0f;
                }
                if constexpr (!PAGED) {
#pragma unroll
                    for (int u = 0; u < 2 * DB; ++u) N::keep(vf[u], mine);
                }
            }
            if (more) {
                if constexpr (kLds) rows.released();
                load_keys(tile + parts);
                load_values(tile + parts);
            }
            if (vis == 0) continue;
            // The reference of the exponentials follows the maximum only when a logit has passed
            // it by more than 8 (of log 2): sums stay below 2^8 * keys, and most steps neither
            // rescale nor look for the maximum across lanes.
            bool grew = false;
            float top[NS];
#pragma unroll
            for (int s = 0; s < NS; ++s) {
                top[s] = x[s][0][0];
#pragma unroll
                for (int j = 1; j < 8; ++j) top[s] = fmaxf(top[s], x[s][j >> 2][j & 3]);
                grew |= top[s] > m[s] + slack;
            }
            if (__any(grew) || far) {
                bool large = false;
#pragma unroll
                for (int s = 0; s < NS; ++s) {
                    const float mn = fmaxf(m[s], max_over_rows(top[s])), from = mn == -kInf ? 0.0f : mn;
                    const float f = __builtin_amdgcn_exp2f((m[s] - from) * sl2);
                    m[s] = mn;
                    ref[s] = from * sl2;
                    large |= fabsf(ref[s]) > kFarExponent;
                    l[s] *= f;
#pragma unroll
                    for (int k = 0; k < 2 * DB; ++k) o[s][k] *= f;
                }
                far = far || __any(large);
                if (__builtin_expect(far, 0)) {
#pragma unroll
                    for (int s = 0; s < NS; ++s) {
                        ref[s] = 0.0f;
#pragma unroll
                        for (int j = 0; j < 8; ++j) x[s][j >> 2][j & 3] -= m[s] == -kInf ? 0.0f : m[s];
                    }
                }
            }
            float p[NS][8];
#pragma unroll
            for (int s = 0; s < NS; ++s) {
                float sum = 0.0f;
#pragma unroll
                for (int j = 0; j < 8; ++j) {
                    p[s][j] = __builtin_amdgcn_exp2f(fmaf(x[s][j >> 2][j & 3], sl2, -ref[s]));
                    sum += p[s][j];
                    if constexpr (PAGED) p[s][j] *= vs[j >> 2][j & 3];
                }
                l[s] += sum;
            }
#pragma unroll
            for (int s = 0; s < NS; ++s) add_weighted<T, TERMS, 2 * DB>(vf, p[s], o[s]);
        }
    }
    SumRef sums[NS];
#pragma unroll
    for (int s = 0; s < NS; ++s) {
        const double rest = far ? static_cast<double>(m[s]) * static_cast<double>(sl2) : ref[s];
        sums[s] = SumRef{offset[s], sum_over_rows(l[s]), m[s] == -kInf ? -static_cast<double>(kInf) : rest};
    }

    // four channels of one row to where they belong
    auto finish = [&](int col, int head, int ch, const SumRef &r, f32x4 x) {
        const int row = q0 + col;
        if (row >= a.Nq) return;
        if (a.nsplit > 1) {
            if (row >= qlen) return;
            const int64_t at = ((static_cast<int64_t>(split) * a.B + b) * a.H + head) * a.Nq + row;
            if (ch < a.D) *(REX_GLOBAL f32x4 *)(a.part + at * a.D + ch) = x;
            if (ch == 0) *(REX_GLOBAL f32x4 *)(a.part_ml + at) = __builtin_bit_cast(f32x4, r);
            return;
        }
        const float inv = r.sum == 0.0f ? 0.0f : 1.0f / r.sum;
#pragma unroll
        for (int i = 0; i < 4; ++i) x[i] = row < qlen ? x[i] * inv : 0.0f;
        const int64_t at = ((static_cast<int64_t>(b) * a.Nq + row) * a.H + head) * a.D + ch;
        if (ch < a.D) {
            N::store4(static_cast<char *>(a.out) + at * N::kSize, x);
            if (a.out_f32) *(REX_GLOBAL f32x4 *)(a.out_f32 + at) = x;
        }
        if (ch == 0 && a.lse)
            as_global_mut<float>(a.lse)[(static_cast<int64_t>(b) * a.H + head) * a.Nq + row] =
                row < qlen ? row_lse(r) : -kInf;
    };

    if (parts == 1) {
#pragma unroll
        for (int s = 0; s < NS; ++s)
#pragma unroll
            for (int u = 0; u < 2 * DB; ++u)
                finish(16 * s + n, h, quad_channel<kNatural>(u, g), sums[s], quad_values<kNatural>(o[s], u));
        return;
    }
    // The waves of a head meet: what their sums refer to first, then the scaled sums of the values,
    // with that of the weights in the first of a row's four spare places.  A reference is one number
    // in units of log 2, or (+inf, and what it stands for beside it) that of a wave whose logits are far.
    float *near_refs = reinterpret_cast<float *>(smem + lds.near);
    SumRef *far_refs = reinterpret_cast<SumRef *>(smem + lds.ref);
    float *acc = reinterpret_cast<float *>(smem + lds.acc);
    auto join = [&](int head, int col) {
        float top = -kInf;
        for (int p = 0; p < parts; ++p) top = fmaxf(top, near_refs[(p * hp + head) * kCols + col]);
        return top;
    };
    auto join_far = [&](int head, int col) {
        SumRef to = far_refs[head * kCols + col];
        for (int p = 1; p < parts; ++p) reach(to, far_refs[(p * hp + head) * kCols + col]);
        return to;
    };
    __syncthreads();                        // the tables of the loop are overwritten
    if (g == 0) {
#pragma unroll
        for (int s = 0; s < NS; ++s) {
            near_refs[wave * kCols + 16 * s + n] = m[s] == -kInf ? -kInf : far ? kInf : ref[s];
            far_refs[wave * kCols + 16 * s + n] = sums[s];
        }
    }
    __syncthreads();
#pragma unroll
    for (int s = 0; s < NS; ++s) {
        const float top = join(hw, 16 * s + n);
        float f = __builtin_amdgcn_exp2f((m[s] == -kInf ? -kInf : ref[s]) - (top == -kInf ? 0.0f : top));
        if (top == kInf) f = __builtin_amdgcn_exp2f(ref_gap(sums[s], join_far(hw, 16 * s + n)));
        float *dst = acc + (wave * kCols + 16 * s + n) * (kDP + 4);
        if (g == 0) dst[kDP] = sums[s].sum * f;
#pragma unroll
        for (int u = 0; u < 2 * DB; ++u)
            *reinterpret_cast<f32x4 *>(dst + quad_channel<kNatural>(u, g)) = quad_values<kNatural>(o[s], u) * f;
    }
    __syncthreads();
    for (int e = tid; e < hp * kCols * DB * 8; e += kAttnWaves * 64) {
        const int ch = (e % (DB * 8)) * 4, col = (e / (DB * 8)) % kCols, w = e / (DB * 8 * kCols);
        SumRef r{};
        f32x4 x = {};
        if (ch == 0 && (a.lse || a.nsplit > 1)) {
            const float top = join(w, col);
            r.rest = top;
            if (top == kInf) r = join_far(w, col);
        }
        r.sum = 0.0f;
        for (int p = 0; p < parts; ++p) {
            const float *src = acc + ((p * hp + w) * kCols + col) * (kDP + 4);
            r.sum += src[kDP];
            x += *reinterpret_cast<const f32x4 *>(src + ch);
        }
        finish(col, h0 + w, ch, r, x);
    }
}

// Columns of one workgroup: 32 queries, or 16 where there are no more and for heads of more
// than 64 channels, whose sums would fill the registers.
template <typename T, int DB, int NS, bool PAGED, int TERMS>
void run_fwd(const AttnArgs &a, hipStream_t s) {
    const dim3 grid(xcd_grid(a.nwg, a.per)), block(kAttnWaves * 64);
    const FwdLds lds = fwd_lds(16 * NS, 32 * DB, a.hp, a.parts, a.rule.nb, a.bias != nullptr,
                               fwd_tiles<T, DB, PAGED>());
    if (a.bias)
        hipLaunchKernelGGL((attn_fwd_kernel<T, DB, NS, true, PAGED, TERMS>), grid, block, lds.total, s, a);
    else
        hipLaunchKernelGGL((attn_fwd_kernel<T, DB, NS, false, PAGED, TERMS>), grid, block, lds.total, s, a);
}

template <typename T, bool PAGED, int TERMS>
hipError_t run_fwd_sized(const AttnArgs &a, int cols, hipStream_t s) {
    if (a.D <= 32) {
        if (cols == 16) run_fwd<T, 1, 1, PAGED, TERMS>(a, s);
        else run_fwd<T, 1, 2, PAGED, TERMS>(a, s);
    } else if (a.D <= 64) {
        if (cols == 16) run_fwd<T, 2, 1, PAGED, TERMS>(a, s);
        else run_fwd<T, 2, 2, PAGED, TERMS>(a, s);
    } else {
        run_fwd<T, 4, 1, PAGED, TERMS>(a, s);
    }
    return hipGetLastError();
}

}  // namespace rex
