// attn_bwd.hip -- the backward of the attention among boxes (box_attn_bwd).
//
//   dq        query columns, keys streamed: grad_q; and for the key pass each row's log sum in
//             units of log 2 (+inf where the row has no part) and delta = sum_c grad_out * out, for
//             bf16 data as the sum of p dp in binary32: `out` carries the rounding of the weights
//             and its own, which is little in grad_q but would be the bias gradient's largest
//             error (6e-4 of it)
//   dkv       key columns, queries streamed, over the heads that share the key head: grad_k,
//             grad_v and the bias gradient
//   hist      the bias gradient's partial tables added up
//
// Both passes compute the weights again from q, k and the row's log sum (seven products of
// the pair matrix instead of five), which costs less than adding one side's gradient with
// atomics, and every element is written once and in a fixed order.
//
// A log sum far from 0 is no longer exact enough for that: beside an offset of -1e9 (a mask that all
// of a row's keys carry) nothing is left of the sum itself, and weights made from it would be off
// by any factor.  For such rows the query pass first finds the offset, the largest logit and the sum of
// the weights again, in three sweeps of a wave over the keys; that takes about as long as the pass,
// and only waves with such a row do it.
//
// The bias gradient is a histogram of ds by bucket.  Each wave adds into tables of its own
// in LDS: LDS serves a wave's additions in order, so the sums repeat bit for bit.  The tables
// are binary64: an addition of 64 lanes to LDS takes 18 to 30 cycles of a CU there, 193 in
// binary32 (measured, whatever the addresses).
//
// Measured, 16 images of up to 1000 boxes in 16 heads of 64 channels, bf16: dq 262 us, dkv
// 512, hist 5.  dkv has four products of the pair matrix, two of them in two parts, and its operands
// leave two waves on a SIMD; without its histogram it takes 70 % of that.  So what bounds it is LDS (reads of
// rows, biases and buckets, and the histogram: 38 % of the CUs' time, and 12 % of conflicts) and vector
// instructions (40 %) from few waves.  8 heads of 128: 395, 857 and 8 us.  Two images of 512 boxes
// in 8 heads of 32, binary32: 23, 28 and 4 us; of 128: 117, 168 and 4.
#include "attn.hpp"

namespace rex {

namespace {

// Steps whose buckets are computed between two barriers.
inline __host__ __device__ int bwd_ahead(int parts) { return parts >= 2 ? 1 : 2; }

// LDS of the two passes, bytes; `heads` tables of biases (and histograms) a wave.
struct BwdLds {
    int bias, hist, copies, geo, buck, tile, acc, total;
};
inline __host__ __device__ BwdLds bwd_lds(int cols, int dp, int hp, int parts, int heads, int nb,
                                          bool bias, bool hist, int tiles) {
    BwdLds l{};
    int at = 0;
    const int table = (nb * nb * 4 + 15) & ~15;
    l.bias = at;
    if (bias) at += hp * heads * table;
    l.geo = at;
    if (bias) at += cols * 16;
    l.buck = at;
    if (bias) at += 2 * bwd_ahead(parts) * parts * cols * kBuckStride * 2;
    l.tile = at;
    at += kAttnWaves * tiles * kTile * dp * 2;        // each wave's tiles of bf16 rows
    l.hist = at;
    l.copies = 1;                 // copies of a wave's table: a power of two that fits
    if (bias && hist) {
        const int waves = kAttnWaves * heads * nb * nb * 8;
        while (l.copies < 4 && at + 2 * l.copies * waves <= kLdsBytes) l.copies *= 2;
        at += (l.copies * waves + 15) & ~15;
    }
    l.acc = 0;                    // the end: the tables are no longer needed
    const int end = parts > 1 ? hp * parts * cols * (dp + 4) * 4 : 0;
    l.total = at > end ? at : end;
    return l;
}

// Rows whose log sum is this far from 0 get it anew: its rounding, and that of its product with log2 e,
// would be up to 2^-17 of a weight and more.
constexpr float kFarLse = 128.0f;
// Their mark is the last bit of what the key pass is told (2^-24 of a log sum that is near).
__device__ __forceinline__ float mark_row(float lse, bool far) {
    return __uint_as_float((__float_as_uint(lse) & ~1u) | (far ? 1u : 0u));
}
__device__ __forceinline__ bool row_marked(float lse) { return __float_as_uint(lse) & 1u; }

// Tiles of bf16 rows that a wave keeps in LDS.  Query pass: keys and
// values, or keys alone for heads of more than 64 channels.  Key pass: queries and upstream
// gradients; none for more than 64 channels, which would leave no room for the histograms.
template <typename T, int DB> constexpr int dq_tiles() { return sizeof(T) == 4 ? 0 : DB <= 2 ? 2 : 1; }
template <typename T, int DB> constexpr bool dkv_lds() { return sizeof(T) == 2 && DB <= 2; }

template <typename T, int DB, int NS, bool BIAS>
__global__ __launch_bounds__(kAttnWaves * 64, 2) void attn_dq_kernel(AttnArgs a) {
    using N = Num<T>;
    using Frag = typename N::Frag;
    using Pair = typename N::Pair;
    constexpr int kCols = 16 * NS, kDP = 32 * DB;
    constexpr bool kLds = sizeof(T) == 2, kNatural = kLds, kBoth = dq_tiles<T, DB>() == 2;
    extern __shared__ char smem[];
    const int id = xcd_order(blockIdx.x, a.nwg, a.per);
    if (id >= a.nwg) return;
    const int tid = threadIdx.x, lane = tid & 63, n = lane & 15, g = lane >> 4;
    const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int hp = a.hp, parts = a.parts, hw = wave & (hp - 1), kw = wave / hp;
    int rest = id;
    const int q0 = rest % a.tiles * kCols;
    rest /= a.tiles;
    const int hgroups = a.H / hp;
    const int h0 = (rest % hgroups) * hp, b = rest / hgroups;
    const int h = h0 + hw, kh = h / a.group;
    const int nb2 = a.rule.nb * a.rule.nb, table = (nb2 * 4 + 15) & ~15;
    const int ahead = bwd_ahead(parts);
    const BwdLds lds = bwd_lds(kCols, kDP, hp, parts, 1, a.rule.nb, BIAS, false, dq_tiles<T, DB>());

    const int qlen = a.qlen ? min(max(a.qlen[b], 0), a.Nq) : a.Nq;
    const int klen = a.klen ? min(max(a.klen[b], 0), a.Nk) : a.Nk;
    const int t1 = q0 < qlen ? (klen + kTile - 1) / kTile : 0;
    const int cols = min(max(qlen - q0, 0), kCols);       // columns that hold a query
    BoxGeo *geo = reinterpret_cast<BoxGeo *>(smem + lds.geo);
    uint16_t *buck = reinterpret_cast<uint16_t *>(smem + lds.buck);
    const float sl2 = a.scale * kLog2e;
    const char *tab = smem + lds.bias + hw * table;
    const HeadRows kr = head_rows<T>(a.k, b, kh, klen, a.D), vr = head_rows<T>(a.v, b, kh, klen, a.D);
    const TileOffsets<T, DB> koff(kr.sr, n, g, a.D), voff(vr.sr, n, g, a.D);
    const LdsTile<DB> rows(smem + lds.tile + wave * dq_tiles<T, DB>() * LdsTile<DB>::kBytes, lane);
    const typename LdsTile<DB>::Loads kload(kr.sr, lane, a.D), vload(vr.sr, lane, a.D);

    auto fill_buckets = [&](int chunk) {
        const int r = lane & 31;
        for (int i = 0; i < ahead; ++i) {
            const int tile = (chunk * ahead + i) * parts + kw;
            if (tile >= t1) return;
            float kx, ky;
            box_centre(box_load(a.kbox + b * a.kbox_sb + min(tile * kTile + r, a.Nk - 1) * a.kbox_sr), kx, ky);
            uint16_t *dst = buck + (((chunk & 1) * ahead + i) * parts + kw) * kCols * kBuckStride + r;
#pragma unroll 2
            for (int c = hw * 2 + (lane >> 5); c < cols; c += 2 * hp)
                dst[c * kBuckStride] = static_cast<uint16_t>(pair_bucket(geo[c], kx, ky, a.rule));
        }
    };

    Frag q[NS][DB], go[NS][DB];
    float lse[NS], delta[NS], sum[NS], natural_lse[NS];
    {
        const HeadRows qr = head_rows<T>(a.q, b, h, qlen, a.D), gr = head_rows<T>(a.gout, b, h, qlen, a.D);
        const Rows out{a.fout, a.gout.sb, a.gout.sr, a.gout.sh};
        const int first = min(q0, max(qlen - 1, 0));
        const int64_t bh = static_cast<int64_t>(b) * a.H + h;
        Frag o[NS][DB];
        load_columns<T, DB, NS>(qr.at(first), qr.sr, n, g, a.D, q);
        load_columns<T, DB, NS>(gr.at(first), gr.sr, n, g, a.D, go);
        load_columns<T, DB, NS>(head_rows<T>(out, b, h, qlen, a.D).at(first), gr.sr, n, g, a.D, o);
#pragma unroll
        for (int s = 0; s < NS; ++s) lse[s] = as_global<float>(a.flse)[bh * a.Nq + min(q0 + 16 * s + n, a.Nq - 1)];
#pragma unroll
        for (int s = 0; s < NS; ++s) {
            const int row = q0 + 16 * s + n;
            // out (rows) times grad_out (columns) has delta on its diagonal, summed as dp is: where a
            // row sees one key and out is its value to the last bit, dp - delta is 0
            f32x4 t = {};
#pragma unroll
            for (int k = 0; k < DB; ++k) t = N::mma(o[s][k], go[s][k], t);
            const float mine = n & 2 ? (n & 1 ? t[3] : t[2]) : (n & 1 ? t[1] : t[0]);
            float d = g == n >> 2 ? mine : 0.0f;
            if (!N::kExact && a.fout_f32) {              // of what was not rounded
                d = 0.0f;
                const int64_t at = ((static_cast<int64_t>(b) * a.Nq + min(row, a.Nq - 1)) * a.H + h) * a.D;
#pragma unroll 1
                for (int ch = 8 * g; ch < a.D; ch += 32) {
                    const f32x8 x = Num<float>::load(reinterpret_cast<const char *>(a.fout_f32 + at + ch));
                    const Frag y = N::load(static_cast<const char *>(a.gout.p) + (at + ch) * N::kSize);
#pragma unroll
                    for (int i = 0; i < 8; ++i) d = fmaf(static_cast<float>(y[i]), x[i], d);
                }
            }
            d = sum_over_rows(d);
            const bool none = row >= qlen || lse[s] == -kInf;
            natural_lse[s] = none ? 0.0f : lse[s];
            lse[s] = none ? kInf : mark_row(lse[s] * kLog2e, false);
            delta[s] = none ? 0.0f : d;
            sum[s] = 0.0f;
        }
    }
    const float *const bias = BIAS ? a.bias + static_cast<int64_t>(h) * nb2 : nullptr;
    bool wide = false;                  // (wide_table)
    if (BIAS) {
        for (int i = lane + 64 * kw; i < nb2; i += 64 * parts)
            reinterpret_cast<float *>(smem + lds.bias + hw * table)[i] = table_entry(as_global<float>(bias)[i], a.scale);
        if (tid < cols) geo[tid] = box_geo(box_load(a.qbox + b * a.qbox_sb + (q0 + tid) * a.qbox_sr));
        // columns without a query: bucket 0 of whatever they hold
        if (cols < kCols)
            for (int i = tid; i < 2 * ahead * parts * kCols * kBuckStride / 2; i += kAttnWaves * 64)
                reinterpret_cast<uint32_t *>(buck)[i] = 0u;
        __syncthreads();
        wide = wide_table(tab, nb2, a.scale, lane);
        fill_buckets(0);
    }
    // What far rows' logits are relative to: their largest bias and their largest logit.
    float offset[NS] = {}, peak[NS] = {};
    bool far_rows = false;
#pragma unroll
    for (int s = 0; s < NS; ++s) far_rows |= fabsf(natural_lse[s]) >= kFarLse;
    far_rows = __any(far_rows);
    // what a logit's sum starts with, from an entry of a wide table
    const float per_scale = 1.0f / a.scale;
    auto start = [&](float entry, int s) { return (entry - offset[s]) * per_scale; };
    if (far_rows) {
        float most[NS], most_bias[NS], total[NS];
#pragma unroll
        for (int s = 0; s < NS; ++s) {
            most[s] = most_bias[s] = -kInf;
            total[s] = 0.0f;
        }
        // 0: the largest bias (of wide tables), 1: the largest logit, 2: the sum
        for (int sweep = wide ? 0 : 1; sweep < 3; ++sweep) {
            for (int tile = 0; tile < t1; ++tile) {
                f32x4 sc[NS][2] = {};
                uint32_t on = 0;
#pragma unroll
                for (int j = 0; j < 8; ++j) {
                    const int key = tile * kTile + 8 * g + j, at = min(key, a.Nk - 1);
                    bool live = key < klen;
                    if (a.kmask) live = live && as_global<uint8_t>(a.kmask)[static_cast<int64_t>(b) * a.Nk + at] != 0;
                    on |= live ? 1u << j : 0u;
                    if (BIAS) {
                        float kx, ky;
                        box_centre(box_load(a.kbox + b * a.kbox_sb + at * a.kbox_sr), kx, ky);
#pragma unroll
                        for (int s = 0; s < NS; ++s) {
                            const uint32_t to = pair_bucket(geo[min(16 * s + n, max(cols - 1, 0))], kx, ky, a.rule);
                            sc[s][j >> 2][j & 3] = wide ? wide_entry(bias, to) : *reinterpret_cast<const float *>(tab + to);
                        }
                    }
                }
                Frag kf[2][DB];
                if (sweep > 0) koff.frags(kr.at(tile * kTile), tile * kTile + kTile <= klen, kf);
#pragma unroll
                for (int s = 0; s < NS; ++s)
#pragma unroll
                    for (int j = 0; j < 8; ++j) {
                        const float e = sc[s][j >> 2][j & 3];
                        if (sweep == 0) most_bias[s] = on >> j & 1u ? fmaxf(most_bias[s], e) : most_bias[s];
                        if (wide) sc[s][j >> 2][j & 3] = start(e, s);
                    }
                if (sweep == 0) continue;
#pragma unroll
                for (int s = 0; s < NS; ++s)
#pragma unroll
                    for (int t = 0; t < 2; ++t)
#pragma unroll
                        for (int k = 0; k < DB; ++k) sc[s][t] = N::mma(kf[t][k], q[s][k], sc[s][t]);
#pragma unroll
                for (int s = 0; s < NS; ++s)
#pragma unroll
                    for (int j = 0; j < 8; ++j) {
                        const float e = on >> j & 1u ? sc[s][j >> 2][j & 3] : -kInf;
                        if (sweep == 1) most[s] = fmaxf(most[s], e);
                        else total[s] += __builtin_amdgcn_exp2f((e - peak[s]) * sl2);
                    }
            }
#pragma unroll
            for (int s = 0; s < NS; ++s) {
                const bool is = fabsf(natural_lse[s]) >= kFarLse;
                if (sweep == 0) offset[s] = is ? max_over_rows(most_bias[s]) : 0.0f;
                else if (sweep == 1) peak[s] = is ? max_over_rows(most[s]) : 0.0f;
                else if (is) lse[s] = mark_row(__builtin_amdgcn_logf(sum_over_rows(total[s])), true);
            }
        }
    }
    // for the key pass; delta of bf16 data follows at the end
#pragma unroll
    for (int s = 0; s < NS; ++s) {
        const int row = q0 + 16 * s + n;
        const int64_t at = ((static_cast<int64_t>(b) * a.H + h) * a.Nqp + row) * 2;
        gptr<float> st = as_global_mut<float>(a.rowstat) + at;
        if (kw == 0 && g == 0 && row < a.Nqp) {
            st[0] = lse[s];
            if (N::kExact || row >= qlen) st[1] = delta[s];
            if (far_rows) *(REX_GLOBAL f32x2 *)(a.rowfar + at) = f32x2{offset[s], peak[s]};
            if (n == 0) as_global_mut<int32_t>(a.far)[(static_cast<int64_t>(b) * a.H + h) * (a.Nqp / 16) + row / 16] = far_rows;
        }
        // 16 columns: the rows that fill up the last 32
        if (NS == 1 && kw == 0 && g == 1 && q0 + 16 >= a.Nq && row + 16 < a.Nqp) {
            st[32] = kInf;
            st[33] = 0.0f;
        }
    }
    f32x4 dq[NS][2 * DB] = {};
    const int steps = (t1 + parts - 1) / parts, chunks = (steps + ahead - 1) / ahead;
    for (int chunk = 0; chunk < chunks; ++chunk) {
        if (BIAS) {
            __syncthreads();
            if (chunk + 1 < chunks) fill_buckets(chunk + 1);
        }
        for (int it = 0; it < ahead; ++it) {
            const int tile = (chunk * ahead + it) * parts + kw;
            if (tile >= t1) break;
            const auto rk = kr.at(tile * kTile), rv = vr.at(tile * kTile);
            const bool inside = tile * kTile + kTile <= klen;
            Frag kf[2][DB], vf[2][DB], kt[2 * DB];
            Pair kp[DB][8];
            auto fill = [&](int to) {
                const bool in = to * kTile + kTile <= klen;
                rows.fill(kr.at(to * kTile), in, kload);
                if constexpr (kBoth) rows.fill(vr.at(to * kTile), in, vload, 1);
            };
            if constexpr (kLds) {
                if (it == 0 && chunk == 0) fill(tile);              // later ones: a step ago
                rows.arrived();
                if constexpr (!kBoth) voff.frags(rv, inside, vf);
#pragma unroll
                for (int t = 0; t < 2; ++t)
#pragma unroll
                    for (int k = 0; k < DB; ++k) {
                        kf[t][k] = rows.rows(t, k);
                        if constexpr (kBoth) vf[t][k] = rows.rows(t, k, 1);
                    }
#pragma unroll
                for (int u = 0; u < 2 * DB; ++u) kt[u] = rows.channels(u);
            } else {
                koff.frags(rk, inside, kf);
                voff.frags(rv, inside, vf);
                koff.pairs(rk, inside, kp);
            }
            const int key = tile * kTile + (lane & 31);
            bool on = key < klen;
            if (a.kmask)
                on = on && as_global<uint8_t>(a.kmask)[static_cast<int64_t>(b) * a.Nk + min(key, a.Nk - 1)] != 0;
            const uint32_t vis = static_cast<uint32_t>(__ballot(on));
            const uint16_t *bk = buck + ((((chunk & 1) * ahead + it) * parts + kw) * kCols + n) * kBuckStride + 8 * g;
            f32x4 sc[NS][2], dp[NS][2];
#pragma unroll
            for (int s = 0; s < NS; ++s) {
                sc[s][0] = sc[s][1] = f32x4{};
                if (BIAS) table_gather(*reinterpret_cast<const u32x4 *>(bk + 16 * s * kBuckStride), tab, sc[s]);
            }
            float x[NS][8];
#pragma unroll
            for (int t = 0; t < 2; ++t)
#pragma unroll
                for (int s = 0; s < NS; ++s) {
                    dp[s][t] = f32x4{};
#pragma unroll
                    for (int k = 0; k < DB; ++k) {
                        sc[s][t] = N::mma(kf[t][k], q[s][k], sc[s][t]);
                        dp[s][t] = N::mma(vf[t][k], go[s][k], dp[s][t]);
                    }
#pragma unroll
                    for (int i = 0; i < 4; ++i) {
                        const float p = __builtin_amdgcn_exp2f(fmaf(sc[s][t][i], sl2, -lse[s]));
                        x[s][4 * t + i] = p * (dp[s][t][i] - delta[s]);
                        dp[s][t][i] *= p;
                    }
                }
            if constexpr (!kLds) {
#pragma unroll
                for (int k = 0; k < DB; ++k) N::split(kp[k], kt[2 * k], kt[2 * k + 1]);
            }
            if (vis != 0xffffffffu || __builtin_expect(wide || far_rows, 0)) {
                const uint32_t mine = vis >> (8 * g);
                if (__builtin_expect(wide || far_rows, 0)) {   // all of it anew, as the sweeps made their logits
                    Frag ka[2][DB], va[2][DB];
                    if constexpr (kLds) {
#pragma unroll
                        for (int t = 0; t < 2; ++t)
#pragma unroll
                            for (int k = 0; k < DB; ++k) {
                                ka[t][k] = rows.rows(t, k);
                                if constexpr (kBoth) va[t][k] = rows.rows(t, k, 1);
                            }
                    } else {
                        koff.frags(rk, inside, ka);
                    }
                    if constexpr (!kBoth) voff.frags(rv, inside, va);
#pragma unroll
                    for (int s = 0; s < NS; ++s) {
                        sc[s][0] = sc[s][1] = f32x4{};
                        if (BIAS) {
                            const u32x4 to = *reinterpret_cast<const u32x4 *>(bk + 16 * s * kBuckStride);
                            if (wide) {
                                wide_gather(to, bias, sc[s]);
#pragma unroll
                                for (int j = 0; j < 8; ++j) sc[s][j >> 2][j & 3] = start(sc[s][j >> 2][j & 3], s);
                            } else {
                                table_gather(to, tab, sc[s]);
                            }
                        }
                    }
                    // No condition among the products: the compiler (ROCm 7.2) leaves out the wait for a
                    // product's result where its first use stands behind a block that may be skipped.
#pragma unroll
                    for (int s = 0; s < NS; ++s) {
#pragma unroll
                        for (int t = 0; t < 2; ++t) {
                            dp[s][t] = f32x4{};
#pragma unroll
                            for (int k = 0; k < DB; ++k) {
                                sc[s][t] = N::mma(ka[t][k], q[s][k], sc[s][t]);
                                dp[s][t] = N::mma(va[t][k], go[s][k], dp[s][t]);
                            }
#pragma unroll
                            for (int i = 0; i < 4; ++i) {
                                const float p = __builtin_amdgcn_exp2f(fmaf(sc[s][t][i] - peak[s], sl2, -lse[s]));
                                x[s][4 * t + i] = p * (dp[s][t][i] - delta[s]);
                                dp[s][t][i] *= p;
                            }
                        }
                    }
                }
#pragma unroll
                for (int j = 0; j < 8; ++j)
#pragma unroll
                    for (int s = 0; s < NS; ++s) {
                        x[s][j] = mine >> j & 1u ? x[s][j] : 0.0f;
                        dp[s][j >> 2][j & 3] = mine >> j & 1u ? dp[s][j >> 2][j & 3] : 0.0f;
                    }
#pragma unroll
                for (int u = 0; u < 2 * DB; ++u) N::keep(kt[u], mine);
            }
            if (kLds && tile + parts < t1) {
                rows.released();
                fill(tile + parts);
            }
            if (!N::kExact) {
#pragma unroll
                for (int s = 0; s < NS; ++s)
#pragma unroll
                    for (int j = 0; j < 8; ++j) sum[s] += dp[s][j >> 2][j & 3];
            }
#pragma unroll
            for (int s = 0; s < NS; ++s) add_weighted<T, 2, 2 * DB>(kt, x[s], dq[s]);
        }
    }
    auto finish = [&](int col, int head, int ch, f32x4 x) {
        const int row = q0 + col;
        if (row >= a.Nq || ch >= a.D) return;
#pragma unroll
        for (int i = 0; i < 4; ++i) x[i] = row < qlen ? x[i] * a.scale : 0.0f;
        N::store4(static_cast<char *>(a.gq) +
                      (((static_cast<int64_t>(b) * a.Nq + row) * a.H + head) * a.D + ch) * N::kSize, x);
    };
    auto keep_delta = [&](int col, int head, float d) {
        if (!N::kExact && q0 + col < qlen)
            as_global_mut<float>(a.rowstat)[((static_cast<int64_t>(b) * a.H + head) * a.Nqp + q0 + col) * 2 + 1] = d;
    };
#pragma unroll
    for (int s = 0; s < NS; ++s) sum[s] = sum_over_rows(sum[s]);
    if (parts == 1) {
#pragma unroll
        for (int s = 0; s < NS; ++s) {
            if (g == 0) keep_delta(16 * s + n, h, sum[s]);
#pragma unroll
            for (int u = 0; u < 2 * DB; ++u)
                finish(16 * s + n, h, quad_channel<kNatural>(u, g), quad_values<kNatural>(dq[s], u));
        }
        return;
    }
    // the parts' sums; the first of a row's four spare places holds its sum of p dp
    float *acc = reinterpret_cast<float *>(smem + lds.acc);
    __syncthreads();
#pragma unroll
    for (int s = 0; s < NS; ++s) {
        float *dst = acc + (wave * kCols + 16 * s + n) * (kDP + 4);
        if (g == 0) dst[kDP] = sum[s];
#pragma unroll
        for (int u = 0; u < 2 * DB; ++u)
            *reinterpret_cast<f32x4 *>(dst + quad_channel<kNatural>(u, g)) = quad_values<kNatural>(dq[s], u);
    }
    __syncthreads();
    for (int e = tid; e < hp * kCols * DB * 8; e += kAttnWaves * 64) {
        const int ch = (e % (DB * 8)) * 4, col = (e / (DB * 8)) % kCols, w = e / (DB * 8 * kCols);
        f32x4 y = {};
        float d = 0.0f;
        for (int p = 0; p < parts; ++p) {
            const float *src = acc + ((p * hp + w) * kCols + col) * (kDP + 4);
            y += *reinterpret_cast<const f32x4 *>(src + ch);
            d += src[kDP];
        }
        if (ch == 0) keep_delta(col, h0 + w, d);
        finish(col, h0 + w, ch, y);
    }
}

template <typename T, int DB, int NS, bool BIAS>
__global__ __launch_bounds__(kAttnWaves * 64, 2) void attn_dkv_kernel(AttnArgs a) {
    using N = Num<T>;
    using Frag = typename N::Frag;
    using Pair = typename N::Pair;
    constexpr int kCols = 16 * NS, kDP = 32 * DB;
    constexpr bool kLds = dkv_lds<T, DB>(), kNatural = kLds;
    extern __shared__ char smem[];
    const int id = xcd_order(blockIdx.x, a.nwg, a.per);
    if (id >= a.nwg) return;
    const int tid = threadIdx.x, lane = tid & 63, n = lane & 15, g = lane >> 4;
    const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int hp = a.hp, parts = a.parts, hw = wave & (hp - 1), kw = wave / hp;
    int rest = id;
    const int sp = rest % a.spans;
    rest /= a.spans;
    const int hgroups = a.Hkv / hp;
    const int kh0 = (rest % hgroups) * hp, b = rest / hgroups;
    const int kh = kh0 + hw;
    const int nb2 = a.rule.nb * a.rule.nb, table = (nb2 * 4 + 15) & ~15;
    const int ahead = bwd_ahead(parts);
    const BwdLds lds = bwd_lds(kCols, kDP, hp, parts, a.head_step, a.rule.nb, BIAS, true, kLds ? 2 : 0);

    const int qlen = a.qlen ? min(max(a.qlen[b], 0), a.Nq) : a.Nq;
    const int klen = a.klen ? min(max(a.klen[b], 0), a.Nk) : a.Nk;
    f32x2 *ctr = reinterpret_cast<f32x2 *>(smem + lds.geo);
    uint16_t *buck = reinterpret_cast<uint16_t *>(smem + lds.buck);
    const float sl2 = a.scale * kLog2e, per_scale = 1.0f / a.scale;
    // entry off / 4 of the lane's copy of table c is at hist + c * nb2 * 8 * copies + off * 2 * copies
    const int copies = lds.copies, log_copies = 32 - __builtin_clz(copies);
    double *const tables = reinterpret_cast<double *>(smem + lds.hist) + wave * a.head_step * nb2 * copies;
    char *const hist = reinterpret_cast<char *>(tables + (n & (copies - 1)));
    float *const partial = BIAS ? a.hist + (static_cast<int64_t>(b) * a.spans + sp) * a.H * nb2 : nullptr;
    const TileOffsets<T, DB> qoff(a.q.sr, n, g, a.D), goff(a.gout.sr, n, g, a.D);
    // queries, then upstream gradients
    const LdsTile<DB> rows(smem + lds.tile + wave * 2 * LdsTile<DB>::kBytes, lane);
    const typename LdsTile<DB>::Loads qload(a.q.sr, lane, a.D), gload(a.gout.sr, lane, a.D);

    const int first_tile = sp * a.span, last_tile = min(first_tile + a.span, a.tiles);
    for (int tile_k = first_tile; tile_k < last_tile; ++tile_k) {
        const int k0 = tile_k * kCols;
        const int cols = min(max(klen - k0, 0), kCols);   // columns that hold a key
        const int t1 = k0 < klen ? (qlen + kTile - 1) / kTile : 0;
        // The key columns.  A masked key's column is whatever its row makes of it: its weights
        // are set to 0 before they reach the histogram, no other column sees them, and zeros
        // are written for it at the end.
        Frag kf[NS][DB], vf[NS][DB];
        bool live[NS];
        {
            const HeadRows kr = head_rows<T>(a.k, b, kh, klen, a.D), vr = head_rows<T>(a.v, b, kh, klen, a.D);
            const int first = min(k0, max(klen - 1, 0));
            load_columns<T, DB, NS>(kr.at(first), kr.sr, n, g, a.D, kf);
            load_columns<T, DB, NS>(vr.at(first), vr.sr, n, g, a.D, vf);
#pragma unroll
            for (int s = 0; s < NS; ++s) {
                const int key = k0 + 16 * s + n;
                live[s] = key < klen;
                if (a.kmask)
                    live[s] = live[s] && as_global<uint8_t>(a.kmask)[static_cast<int64_t>(b) * a.Nk + min(key, a.Nk - 1)] != 0;
            }
        }
        bool all_live = true;
#pragma unroll
        for (int s = 0; s < NS; ++s) all_live = all_live && live[s];
        const bool whole = __all(all_live);
        if (BIAS) {
            __syncthreads();              // the last tile's tables have been read
            if (tid < cols) {
                float cx, cy;
                box_centre(box_load(a.kbox + b * a.kbox_sb + (k0 + tid) * a.kbox_sr), cx, cy);
                ctr[tid] = f32x2{cx, cy};
            }
            // columns without a key: bucket 0, to which their zeros are added
            if (cols < kCols)
                for (int i = tid; i < 2 * ahead * parts * kCols * kBuckStride / 2; i += kAttnWaves * 64)
                    reinterpret_cast<uint32_t *>(buck)[i] = 0u;
        }
        // here the streamed side is the queries: row r of the tile is query 32 * tile + r
        auto fill_buckets = [&](int chunk) {
            const int r = lane & 31;
            for (int i = 0; i < ahead; ++i) {
                const int tile = (chunk * ahead + i) * parts + kw;
                if (tile >= t1) return;
                const BoxGeo q = box_geo(box_load(a.qbox + b * a.qbox_sb + min(tile * kTile + r, a.Nq - 1) * a.qbox_sr));
                uint16_t *dst = buck + (((chunk & 1) * ahead + i) * parts + kw) * kCols * kBuckStride + r;
#pragma unroll 2
                for (int c = hw * 2 + (lane >> 5); c < cols; c += 2 * hp)
                    dst[c * kBuckStride] = static_cast<uint16_t>(pair_bucket(q, ctr[c][0], ctr[c][1], a.rule));
            }
        };

        f32x4 dk[NS][2 * DB] = {}, dv[NS][2 * DB] = {}, st_next[4];
        const int steps = (t1 + parts - 1) / parts, chunks = (steps + ahead - 1) / ahead;
        uint32_t wides = 0, special = 0;  // heads of these whose tables are wide; and those with far rows
        for (int first = 0; first < a.group; first += a.head_step) {
            const int many = min(a.head_step, a.group - first);
            special = 0;
            for (int c = 0; c < many; ++c) {
                gcptr<int32_t> far = as_global<int32_t>(a.far) + (static_cast<int64_t>(b) * a.H + kh * a.group + first + c) * (a.Nqp / 16);
                bool some = false;
                for (int i = lane; i < (a.Nq + 15) / 16; i += 64) some |= far[i] != 0;
                special |= __any(some) ? 1u << c : 0u;
            }
            if (BIAS) {
                __syncthreads();          // the tables of the last heads have been read
                for (int c = 0; c < many; ++c)
                    for (int i = lane + 64 * kw; i < nb2; i += 64 * parts)
                        reinterpret_cast<float *>(smem + lds.bias + (hw * a.head_step + c) * table)[i] =
                            table_entry(as_global<float>(a.bias)[static_cast<int64_t>(kh * a.group + first + c) * nb2 + i], a.scale);
                for (int i = lane; i < many * nb2 * copies; i += 64) tables[i] = 0.0;
                fill_buckets(0);
            }
            for (int chunk = 0; chunk < chunks; ++chunk) {
                if (BIAS) {
                    __syncthreads();
                    if (chunk == 0) {
                        wides = 0;
                        for (int c = 0; c < many; ++c)
                            wides |= wide_table(smem + lds.bias + (hw * a.head_step + c) * table, nb2, a.scale, lane) ? 1u << c : 0u;
                        special |= wides;
                    }
                    if (chunk + 1 < chunks) fill_buckets(chunk + 1);
                }
                for (int it = 0; it < ahead; ++it) {
                    const int tile = (chunk * ahead + it) * parts + kw;
                    if (tile >= t1) break;
                    const uint16_t *bk = buck + ((((chunk & 1) * ahead + it) * parts + kw) * kCols + n) * kBuckStride + 8 * g;
                    for (int c = 0; c < many; ++c) {
                        const int h = kh * a.group + first + c;
                        const char *tab = smem + lds.bias + (hw * a.head_step + c) * table;
                        const auto rq = head_rows<T>(a.q, b, h, qlen, a.D).at(tile * kTile);
                        const auto rg = head_rows<T>(a.gout, b, h, qlen, a.D).at(tile * kTile);
                        const bool inside = tile * kTile + kTile <= qlen;
                        // the next head of this tile, or the first of the next tile
                        const bool last = c + 1 == many;
                        const int next = last ? tile + parts : tile, nh = last ? kh * a.group + first : h + 1;
                        auto fill = [&](int to, int head) {
                            const bool in = to * kTile + kTile <= qlen;
                            rows.fill(head_rows<T>(a.q, b, head, qlen, a.D).at(to * kTile), in, qload);
                            rows.fill(head_rows<T>(a.gout, b, head, qlen, a.D).at(to * kTile), in, gload, 1);
                        };
                        auto load_stat = [&](int to, int head, f32x4 (&x)[4]) {
                            const float *p = a.rowstat + ((static_cast<int64_t>(b) * a.H + head) * a.Nqp + to * kTile + 8 * g) * 2;
#pragma unroll
                            for (int i = 0; i < 4; ++i) x[i] = *(const REX_GLOBAL f32x4 *)(p + 4 * i);
                        };
                        f32x4 st[4];                  // (log sum, delta) of the lane's eight rows
                        if constexpr (kLds) {
                            if (c == 0 && it == 0 && chunk == 0) {         // later ones: a step ago
                                rows.released();
                                fill(tile, h);
                                load_stat(tile, h, st_next);
                            }
                            rows.arrived();
#pragma unroll
                            for (int i = 0; i < 4; ++i) st[i] = st_next[i];
                            if (next < t1) load_stat(next, nh, st_next);
                        } else {
                            load_stat(tile, h, st);
                        }
                        u32x4 at[NS];
                        f32x4 sc[NS][2];
#pragma unroll
                        for (int s = 0; s < NS; ++s) {
                            sc[s][0] = sc[s][1] = f32x4{};
                            at[s] = u32x4{};
                            if (BIAS) {
                                at[s] = *reinterpret_cast<const u32x4 *>(bk + 16 * s * kBuckStride);
                                table_gather(at[s], tab, sc[s]);
                            }
                        }
                        // heads of wide tables or with far rows: what a row's logits are relative to
                        const bool other = special >> c & 1u;
                        f32x4 peak[2] = {};
                        if (__builtin_expect(other, 0)) {
                            const bool wide = wides >> c & 1u;
                            const float *from = a.rowfar + ((static_cast<int64_t>(b) * a.H + h) * a.Nqp + tile * kTile + 8 * g) * 2;
                            if (BIAS && wide) {
#pragma unroll
                                for (int s = 0; s < NS; ++s) wide_gather(at[s], a.bias + static_cast<int64_t>(h) * nb2, sc[s]);
                            }
#pragma unroll
                            for (int j = 0; j < 8; ++j) {
                                f32x2 x = {};
                                if (row_marked(st[j >> 1][2 * (j & 1)])) x = *(const REX_GLOBAL f32x2 *)(from + 2 * j);
                                peak[j >> 2][j & 3] = x[1];
#pragma unroll
                                for (int s = 0; s < NS; ++s)
                                    if (wide) sc[s][j >> 2][j & 3] = (sc[s][j >> 2][j & 3] - x[0]) * per_scale;
                            }
                        }
                        float pr[NS][8], ds[NS][8];
                        Frag qf[2][DB], gf[2][DB];
                        if constexpr (!kLds) {
                            qoff.frags(rq, inside, qf);
                            goff.frags(rg, inside, gf);
                        }
#pragma unroll
                        for (int t = 0; t < 2; ++t) {
                            if constexpr (kLds) {
#pragma unroll
                                for (int k = 0; k < DB; ++k) {
                                    qf[t][k] = rows.rows(t, k);
                                    gf[t][k] = rows.rows(t, k, 1);
                                }
                            }
#pragma unroll
                            for (int s = 0; s < NS; ++s) {
                                f32x4 dp = {};
#pragma unroll
                                for (int k = 0; k < DB; ++k) {
                                    sc[s][t] = N::mma(qf[t][k], kf[s][k], sc[s][t]);
                                    dp = N::mma(gf[t][k], vf[s][k], dp);
                                }
                                // 0 in most rows, but no condition here: the compiler (ROCm 7.2) leaves out
                                // the wait for sc where a block that may be skipped stands before its use
                                sc[s][t] -= peak[t];
#pragma unroll
                                for (int i = 0; i < 4; ++i) {
                                    const f32x4 two = st[2 * t + (i >> 1)];
                                    const float p = __builtin_amdgcn_exp2f(fmaf(sc[s][t][i], sl2, -two[2 * (i & 1)]));
                                    pr[s][4 * t + i] = p;
                                    ds[s][4 * t + i] = p * (dp[i] - two[2 * (i & 1) + 1]);
                                }
                            }
                        }
                        // all additions of a tile in a row: reads of LDS would wait for those
                        // before them
                        if (BIAS) {
                            if (!whole) {
#pragma unroll
                                for (int s = 0; s < NS; ++s)
#pragma unroll
                                    for (int j = 0; j < 8; ++j) ds[s][j] = live[s] ? ds[s][j] : 0.0f;
                            }
                            char *const to = hist + c * nb2 * 8 * copies;
#pragma unroll
                            for (int s = 0; s < NS; ++s) {
#pragma unroll
                                for (int j = 0; j < 8; ++j)
                                    unsafeAtomicAdd(reinterpret_cast<double *>(to + (table_offset(at[s], j) << log_copies)),
                                                    static_cast<double>(ds[s][j]));
                            }
                        }
                        {
                            Frag gt[2 * DB];
                            if constexpr (kLds) {
#pragma unroll
                                for (int u = 0; u < 2 * DB; ++u) gt[u] = rows.channels(u, 1);
                            } else {
                                Pair p[DB][8];
                                goff.pairs(rg, inside, p);
#pragma unroll
                                for (int k = 0; k < DB; ++k) N::split(p[k], gt[2 * k], gt[2 * k + 1]);
                            }
#pragma unroll
                            for (int s = 0; s < NS; ++s) add_weighted<T, 2, 2 * DB>(gt, pr[s], dv[s]);
                        }
                        Frag qt[2 * DB];
                        if constexpr (kLds) {
#pragma unroll
                            for (int u = 0; u < 2 * DB; ++u) qt[u] = rows.channels(u);
                            if (next < t1) {
                                rows.released();
                                fill(next, nh);
                            }
                        } else {
                            Pair p[DB][8];
                            qoff.pairs(rq, inside, p);
#pragma unroll
                            for (int k = 0; k < DB; ++k) N::split(p[k], qt[2 * k], qt[2 * k + 1]);
                        }
#pragma unroll
                        for (int s = 0; s < NS; ++s) add_weighted<T, 2, 2 * DB>(qt, ds[s], dk[s]);
                    }
                }
            }
            if (BIAS) {                   // this workgroup's own partial tables
                __syncthreads();
                for (int e = tid; e < hp * many * nb2; e += kAttnWaves * 64) {
                    const int i = e % nb2, c = e / nb2 % many, w = e / (nb2 * many);
                    double sum = 0.0;
                    for (int p = 0; p < parts; ++p) {
                        const double *t = reinterpret_cast<const double *>(smem + lds.hist) +
                                          (((p * hp + w) * a.head_step + c) * nb2 + i) * copies;
                        for (int x = 0; x < copies; ++x) sum += t[x];
                    }
                    gptr<float> dst = as_global_mut<float>(partial) + ((kh0 + w) * a.group + first + c) * nb2 + i;
                    *dst = static_cast<float>(sum) + (tile_k > first_tile ? *dst : 0.0f);
                }
            }
        }

        auto finish = [&](char *out, float f, int col, int head, int ch, f32x4 x) {
            const int key = k0 + col;
            if (key >= a.Nk || ch >= a.D) return;
            bool on = key < klen;
            if (a.kmask && on) on = as_global<uint8_t>(a.kmask)[static_cast<int64_t>(b) * a.Nk + key] != 0;
#pragma unroll
            for (int i = 0; i < 4; ++i) x[i] = on ? x[i] * f : 0.0f;
            N::store4(out + (((static_cast<int64_t>(b) * a.Nk + key) * a.Hkv + head) * a.D + ch) * N::kSize, x);
        };
        auto write = [&](const f32x4 (&d)[NS][2 * DB], char *out, float f) {
            if (parts == 1) {
#pragma unroll
                for (int s = 0; s < NS; ++s)
#pragma unroll
                    for (int u = 0; u < 2 * DB; ++u)
                        finish(out, f, 16 * s + n, kh, quad_channel<kNatural>(u, g), quad_values<kNatural>(d[s], u));
                return;
            }
            float *acc = reinterpret_cast<float *>(smem + lds.acc);
            __syncthreads();
#pragma unroll
            for (int s = 0; s < NS; ++s)
#pragma unroll
                for (int u = 0; u < 2 * DB; ++u)
                    *reinterpret_cast<f32x4 *>(acc + (wave * kCols + 16 * s + n) * (kDP + 4) + quad_channel<kNatural>(u, g)) =
                        quad_values<kNatural>(d[s], u);
            __syncthreads();
            for (int e = tid; e < hp * kCols * DB * 8; e += kAttnWaves * 64) {
                const int ch = (e % (DB * 8)) * 4, col = (e / (DB * 8)) % kCols, w = e / (DB * 8 * kCols);
                f32x4 y = {};
                for (int p = 0; p < parts; ++p)
                    y += *reinterpret_cast<const f32x4 *>(acc + ((p * hp + w) * kCols + col) * (kDP + 4) + ch);
                finish(out, f, col, kh0 + w, ch, y);
            }
        };
        write(dk, static_cast<char *>(a.gk), a.scale);
        write(dv, static_cast<char *>(a.gv), 1.0f);
    }
}

// gbias[h][i] = sum over the partial tables, 16 slices of them side by side, in order.
__global__ __launch_bounds__(1024) void attn_hist_kernel(AttnArgs a) {
    __shared__ float part[16][64];
    const int64_t n = static_cast<int64_t>(a.H) * a.rule.nb * a.rule.nb;
    const int64_t i = static_cast<int64_t>(blockIdx.x) * 64 + (threadIdx.x & 63);
    const int slice = threadIdx.x >> 6;
    float sum = 0.0f;
    if (i < n) {
        gcptr<float> src = as_global<float>(a.hist);
        const int chunks = a.B * a.spans;
#pragma unroll 8
        for (int c = slice; c < chunks; c += 16) sum += src[c * n + i];
    }
    part[slice][threadIdx.x & 63] = sum;
    __syncthreads();
    if (slice == 0 && i < n) {
        for (int s = 1; s < 16; ++s) sum += part[s][threadIdx.x];
        as_global_mut<float>(a.gbias)[i] = sum;
    }
}

template <typename T, int DB, int NS>
void run_pass(const AttnArgs &a, bool keys, hipStream_t s) {
    if (a.nwg == 0) return;
    const dim3 grid(xcd_grid(a.nwg, a.per)), block(kAttnWaves * 64);
    const bool bias = a.bias != nullptr;
    const BwdLds lds = bwd_lds(16 * NS, 32 * DB, a.hp, a.parts, keys ? a.head_step : 1, a.rule.nb,
                               bias, keys, !keys ? dq_tiles<T, DB>() : dkv_lds<T, DB>() ? 2 : 0);
    if (keys && bias)
        hipLaunchKernelGGL((attn_dkv_kernel<T, DB, NS, true>), grid, block, lds.total, s, a);
    else if (keys)
        hipLaunchKernelGGL((attn_dkv_kernel<T, DB, NS, false>), grid, block, lds.total, s, a);
    else if (bias)
        hipLaunchKernelGGL((attn_dq_kernel<T, DB, NS, true>), grid, block, lds.total, s, a);
    else
        hipLaunchKernelGGL((attn_dq_kernel<T, DB, NS, false>), grid, block, lds.total, s, a);
}

template <typename T>
void run_sized(const AttnArgs &a, bool keys, int cols, hipStream_t s) {
    if (a.D <= 32) {
        if (cols == 16) run_pass<T, 1, 1>(a, keys, s);
        else run_pass<T, 1, 2>(a, keys, s);
    } else if (a.D <= 64) {
        if (cols == 16) run_pass<T, 2, 1>(a, keys, s);
        else run_pass<T, 2, 2>(a, keys, s);
    } else {
        run_pass<T, 4, 1>(a, keys, s);
    }
}

void run_typed(const AttnArgs &a, int dtype, bool keys, int cols, hipStream_t s) {
    if (dtype == kF32) run_sized<float>(a, keys, cols, s);
    else run_sized<uint16_t>(a, keys, cols, s);
}

}  // namespace

bool dkv_fits(const AttnArgs &a, int dtype, int cols) {
    const int db = a.D <= 32 ? 1 : a.D <= 64 ? 2 : 4, tiles = dtype == kBF16 && db <= 2 ? 2 : 0;
    return bwd_lds(cols, 32 * db, a.hp, a.parts, a.head_step, a.rule.nb, a.bias != nullptr, true, tiles).total <= kLdsBytes;
}

hipError_t launch_attn_bwd(const AttnArgs &dq, const AttnArgs &dkv, int dtype, int dq_cols,
                           int dkv_cols, hipStream_t s) {
    run_typed(dq, dtype, false, dq_cols, s);
    run_typed(dkv, dtype, true, dkv_cols, s);
    if (dkv.bias) {
        const int64_t t = static_cast<int64_t>(dkv.H) * dkv.rule.nb * dkv.rule.nb;
        hipLaunchKernelGGL(attn_hist_kernel, dim3(static_cast<uint32_t>((t + 63) / 64)), dim3(1024), 0,
                           s, dkv);
    }
    return hipGetLastError();
}

}  // namespace rex
