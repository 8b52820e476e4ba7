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
// share of the products: the workgroup computes each tile's buckets once, a few steps ahead,
// into LDS (16 bits a pair: the byte offset into a head's table, which is in LDS too).
#pragma once

#include "attn.hpp"
#ifndef REX_FWPE
#define REX_FWPE 2
#endif

namespace rex {

// What is in LDS, in bytes from its start.
struct FwdLds {
    int bias, geo, buck, ml, acc, total;
};
// Steps whose buckets are computed between two barriers.
inline __host__ __device__ int fwd_ahead(int parts) { return parts >= 4 ? 1 : 4 / parts; }
inline __host__ __device__ FwdLds fwd_lds(int cols, int dp, int hp, int parts, int nb, bool bias) {
    FwdLds l{};
    int at = 0;
    l.bias = at;
    if (bias) at += (hp * nb * nb * 4 + 15) & ~15;
    l.geo = at;
    if (bias) at += cols * 16;
    l.buck = at;
    if (bias) at += 2 * fwd_ahead(parts) * parts * cols * kBuckStride * 2;
    const int loop = at;
    at = 0;                       // the end: the loop's tables are no longer needed
    l.ml = at;
    if (parts > 1) at += hp * parts * cols * 8;
    l.acc = at;
    if (parts > 1) at += hp * parts * cols * (dp + 4) * 4;
    l.total = at > loop ? at : loop;
    return l;
}

template <typename T, int DB, int NS, bool BIAS, bool PAGED, int TERMS>
__global__ __launch_bounds__(kAttnWaves * 64, REX_FWPE) void attn_fwd_kernel(AttnArgs a) {
    using N = Num<T>;
    using Frag = typename N::Frag;
    using Pair = typename N::Pair;
    constexpr int kCols = 16 * NS, kDP = 32 * DB;
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
    const FwdLds lds = fwd_lds(kCols, kDP, hp, parts, a.rule.nb, BIAS);

    const int qlen = a.qlen ? min(max(a.qlen[b], 0), a.Nq) : a.Nq;
    const int klen = a.klen ? min(max(a.klen[b], 0), a.Nk) : a.Nk;
    const int q0 = tile_q * kCols;
    const int all = (klen + kTile - 1) / kTile;
    const int per = (all + a.nsplit - 1) / a.nsplit;
    const int t0 = min(split * per, all), t1 = q0 < qlen ? min(t0 + per, all) : t0;

    BoxGeo *geo = reinterpret_cast<BoxGeo *>(smem + lds.geo);
    uint16_t *buck = reinterpret_cast<uint16_t *>(smem + lds.buck);
    if (BIAS) {
        const int nb2 = a.rule.nb * a.rule.nb;
        float *t = reinterpret_cast<float *>(smem + lds.bias);
        gcptr<float> src = as_global<float>(a.bias + static_cast<int64_t>(h0) * nb2);
        for (int i = tid; i < hp * nb2; i += kAttnWaves * 64) t[i] = table_entry(src[i], a.scale);
        if (tid < kCols)
            geo[tid] = box_geo(as_global<float>(a.qbox + b * a.qbox_sb +
                                                min(q0 + tid, a.Nq - 1) * a.qbox_sr));
    }

    // the queries: column n of NS tiles; rows that are padding are zeros
    Frag q[NS][DB];
    {
        const HeadRows qr = head_rows<T>(a.q, b, h, qlen, a.D);
        const TileOffsets<T, DB> off(qr.sr, n, g, a.D);
        const auto r = qr.at(min(q0, max(qlen - 1, 0)));
#pragma unroll
        for (int s = 0; s < NS; ++s)
#pragma unroll
            for (int k = 0; k < DB; ++k) q[s][k] = N::load(r, off.f[k] + 16 * s * off.sr, 0);
    }

    // One tile's keys and values, its page and the lane's mask byte, read one step ahead.
    const HeadRows kr = head_rows<T>(a.k, b, kh, PAGED ? 0 : klen, a.D);
    const HeadRows vr = head_rows<T>(a.v, b, kh, PAGED ? 0 : klen, a.D);
    const TileOffsets<T, DB> koff(kr.sr, n, g, a.D), voff(vr.sr, n, g, a.D);
    uint32_t kcode[DB], vcode[DB];         // the same inside a page of the memory
#pragma unroll
    for (int k = 0; k < DB; ++k) {
        kcode[k] = 32 * k + 8 * g < a.D ? n * a.D + 32 * k + 8 * g : kBufOOB;
        vcode[k] = 32 * k + 2 * n < a.D ? (32 * k + 2 * n) * kTile + 4 * g : kBufOOB;
    }
    struct {
        Frag f[2][DB];                                   // keys
        Pair p[DB][8];                                   // values
        u32x2 kc[PAGED ? 2 : 1][PAGED ? DB : 1];         // their codes and scales in the memory
        uint32_t vc[PAGED ? DB : 1][2][2];
        f32x4 ks[2], vs[2];
        int64_t ph;
        bool on;
    } next;
    auto page_of = [&](int tile) -> int {
        const int p = a.pages[static_cast<int64_t>(b) * a.max_pages + tile];
        return p >= 0 && p < a.num_pages ? p : -1;
    };
    auto load_keys = [&](int tile) {
        const int key = tile * kTile + (lane & 31);
        next.on = key < klen;
        if constexpr (PAGED) {
            const int page = page_of(tile);
            next.on = next.on && page >= 0;
            next.ph = static_cast<int64_t>(max(page, 0)) * a.Hkv + kh;
            const auto r = make_rsrc(a.mk + next.ph * kTile * a.D, kTile * a.D);
#pragma unroll
            for (int t = 0; t < 2; ++t) {
                next.ks[t] = *(const REX_GLOBAL f32x4 *)(a.mks + next.ph * kTile + 16 * t + 4 * g);
#pragma unroll
                for (int k = 0; k < DB; ++k)
                    next.kc[t][k] = __builtin_amdgcn_raw_buffer_load_b64(r, kcode[k], 16 * t * a.D, 0);
            }
        } else {
            if (a.kmask)
                next.on = next.on && as_global<uint8_t>(a.kmask)[static_cast<int64_t>(b) * a.Nk + min(key, a.Nk - 1)] != 0;
            koff.frags(kr.at(tile * kTile), tile * kTile + kTile <= klen, next.f);
        }
    };
    auto load_values = [&](int tile) {                   // after load_keys of the same tile
        if constexpr (PAGED) {
            const auto r = make_rsrc(a.mv + next.ph * kTile * a.D, kTile * a.D);
#pragma unroll
            for (int t = 0; t < 2; ++t)
                next.vs[t] = *(const REX_GLOBAL f32x4 *)(a.mvs + next.ph * kTile + 16 * t + 4 * g);
#pragma unroll
            for (int k = 0; k < DB; ++k)
#pragma unroll
                for (int t = 0; t < 2; ++t)
#pragma unroll
                    for (int e = 0; e < 2; ++e)
                        next.vc[k][t][e] = __builtin_amdgcn_raw_buffer_load_b32(r, vcode[k] + kTile * t + 16 * e, 0, 0);
        } else {
            voff.pairs(vr.at(tile * kTile), tile * kTile + kTile <= klen, next.p);
        }
    };
    // Buckets of the chunk's tiles against the workgroup's queries, by the waves that read them.
    auto fill_buckets = [&](int chunk) {
        const int r = lane & 31;
        for (int i = 0; i < ahead; ++i) {
            const int tile = t0 + (chunk * ahead + i) * parts + kw;
            if (tile >= t1) return;
            const float *box;
            if constexpr (PAGED) box = a.mbox + (static_cast<int64_t>(max(page_of(tile), 0)) * kTile + r) * 4;
            else box = a.kbox + b * a.kbox_sb + min(tile * kTile + r, a.Nk - 1) * a.kbox_sr;
            float kx, ky;
            box_centre(as_global<float>(box), kx, ky);
            uint16_t *dst = buck + (((chunk & 1) * ahead + i) * parts + kw) * kCols * kBuckStride + r;
#pragma unroll 2
            for (int c = hw * 2 + (lane >> 5); c < kCols; c += 2 * hp)
                dst[c * kBuckStride] = static_cast<uint16_t>(pair_bucket(geo[c], kx, ky, a.rule));
        }
    };

    const float sl2 = a.scale * kLog2e;
    const char *tab = smem + lds.bias + hw * a.rule.nb * a.rule.nb * 4;
    f32x4 o[NS][2 * DB] = {};      // 16-channel tiles 2k, 2k + 1: even and odd channels
    // The running maximum, in units of the products; what exponents are taken from (m in units
    // of log 2, 0 while there is no key); the sum.
    float m[NS], ref[NS], l[NS];
    const float slack = 8.0f / sl2;
#pragma unroll
    for (int s = 0; s < NS; ++s) {
        m[s] = -kInf;
        ref[s] = l[s] = 0.0f;
    }
    const int steps = (t1 - t0 + parts - 1) / parts, chunks = (steps + ahead - 1) / ahead;
    if (t0 + kw < t1) {
        load_keys(t0 + kw);
        load_values(t0 + kw);
    }
    if (BIAS) {
        __syncthreads();
        fill_buckets(0);
    }

    for (int chunk = 0; chunk < chunks; ++chunk) {
        if (BIAS) {
            __syncthreads();
            if (chunk + 1 < chunks) fill_buckets(chunk + 1);
        }
        for (int i = 0; i < ahead; ++i) {
            const int tile = t0 + (chunk * ahead + i) * parts + kw;
            if (tile >= t1) break;
            const uint32_t vis = static_cast<uint32_t>(__ballot(next.on));   // bit r: key r is visible
            const bool more = tile + parts < t1;
            // what a logit starts with: its bias, or nothing
            f32x4 x[NS][2];
            const uint16_t *bk = buck + ((((chunk & 1) * ahead + i) * parts + kw) * kCols + n) * kBuckStride + 4 * g;
#pragma unroll
            for (int s = 0; s < NS; ++s)
#pragma unroll
                for (int t = 0; t < 2; ++t)
                    x[s][t] = BIAS ? table_gather(*reinterpret_cast<const u32x2 *>(bk + 16 * s * kBuckStride + 16 * t), tab)
                                   : f32x4{};
            // column = query n, rows = keys 4g + e of two tiles
#pragma unroll
            for (int t = 0; t < 2; ++t) {
                Frag kf[DB];
#pragma unroll
                for (int k = 0; k < DB; ++k) {
                    if constexpr (PAGED) {
                        N::widen(kf[k], 0, next.kc[t][k][0]);
                        N::widen(kf[k], 4, next.kc[t][k][1]);
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
            Frag vf[2 * DB];
            f32x4 vs[2];
            if constexpr (PAGED) {
#pragma unroll
                for (int t = 0; t < 2; ++t) vs[t] = next.vs[t];
#pragma unroll
                for (int k = 0; k < DB; ++k)
#pragma unroll
                    for (int t = 0; t < 2; ++t) {
                        N::widen(vf[2 * k + t], 0, next.vc[k][t][0]);
                        N::widen(vf[2 * k + t], 4, next.vc[k][t][1]);
                    }
            }
            if (vis != 0xffffffffu) {
#pragma unroll
                for (int j = 0; j < 8; ++j) {
                    const bool on = (vis >> slot_row(g, j)) & 1u;
#pragma unroll
                    for (int s = 0; s < NS; ++s) x[s][j >> 2][j & 3] = on ? x[s][j >> 2][j & 3] : -kInf;
                    if constexpr (PAGED) {
                        vs[j >> 2][j & 3] = on ? vs[j >> 2][j & 3] : 0.0f;
                    } else {
#pragma unroll
                        for (int k = 0; k < DB; ++k) next.p[k][j] = on ? next.p[k][j] : N::no_pair();
                    }
                }
            }
            if constexpr (!PAGED) {
#pragma unroll
                for (int k = 0; k < DB; ++k) N::split(next.p[k], vf[2 * k], vf[2 * k + 1]);
            }
            if (more) {
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
            if (__any(grew)) {
#pragma unroll
                for (int s = 0; s < NS; ++s) {
                    const float mn = fmaxf(m[s], max_over_rows(top[s]));
                    const float f = __builtin_amdgcn_exp2f((m[s] - (mn == -kInf ? 0.0f : mn)) * sl2);
                    m[s] = mn;
                    ref[s] = mn == -kInf ? 0.0f : mn * sl2;
                    l[s] *= f;
#pragma unroll
                    for (int k = 0; k < 2 * DB; ++k) o[s][k] *= f;
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
#pragma unroll
    for (int s = 0; s < NS; ++s) {
        l[s] = sum_over_rows(l[s]);
        m[s] = m[s] == -kInf ? -kInf : ref[s];       // from here on in units of log 2
    }

    // eight channels of one row, scaled, to where they belong
    auto finish = [&](int col, int head, int ch, float mx, float sum, const float (&x)[8]) {
        const int row = q0 + col;
        if (row >= a.Nq) return;
        if (a.nsplit > 1) {
            if (row >= qlen) return;
            const int64_t at = ((static_cast<int64_t>(split) * a.B + b) * a.H + head) * a.Nq + row;
            if (ch < a.D) Num<float>::store(reinterpret_cast<char *>(a.part + at * a.D + ch), x);
            if (ch == 0) *(REX_GLOBAL f32x2 *)(a.part_ml + at * 2) = f32x2{mx, sum};
            return;
        }
        const float inv = sum == 0.0f ? 0.0f : 1.0f / sum;
        float y[8];
#pragma unroll
        for (int i = 0; i < 8; ++i) y[i] = row < qlen ? x[i] * inv : 0.0f;
        const int64_t at = (((static_cast<int64_t>(b) * a.Nq + row) * a.H + head) * a.D + ch) * N::kSize;
        if (ch < a.D) {
            N::store(static_cast<char *>(a.out) + at, y);
            if (a.out_f32)
                Num<float>::store(reinterpret_cast<char *>(a.out_f32) + at * (4 / N::kSize), y);
        }
        if (ch == 0 && a.lse)
            as_global_mut<float>(a.lse)[(static_cast<int64_t>(b) * a.H + head) * a.Nq + row] =
                row < qlen && sum != 0.0f ? (mx + log2f(sum)) * kLn2 : -kInf;
    };

    if (parts == 1) {
#pragma unroll
        for (int s = 0; s < NS; ++s)
#pragma unroll
            for (int k = 0; k < DB; ++k) {
                float x[8];
#pragma unroll
                for (int i = 0; i < 8; ++i) x[i] = o[s][2 * k + (i & 1)][i >> 1];
                finish(16 * s + n, h, 32 * k + 8 * g, m[s], l[s], x);
            }
        return;
    }
    // The waves of a head meet: maxima and sums first, then the scaled sums of the values.
    f32x2 *ml = reinterpret_cast<f32x2 *>(smem + lds.ml);
    float *acc = reinterpret_cast<float *>(smem + lds.acc);
    __syncthreads();                        // the tables of the loop are overwritten
    if (g == 0) {
#pragma unroll
        for (int s = 0; s < NS; ++s) ml[wave * kCols + 16 * s + n] = f32x2{m[s], l[s]};
    }
    __syncthreads();
#pragma unroll
    for (int s = 0; s < NS; ++s) {
        float mx = -kInf;
        for (int p = 0; p < parts; ++p) mx = fmaxf(mx, ml[(p * hp + hw) * kCols + 16 * s + n][0]);
        const float f = __builtin_amdgcn_exp2f(m[s] - (mx == -kInf ? 0.0f : mx));
#pragma unroll
        for (int k = 0; k < DB; ++k) {
            float *dst = acc + (wave * kCols + 16 * s + n) * (kDP + 4) + 32 * k + 8 * g;
#pragma unroll
            for (int i = 0; i < 8; i += 4)
                *reinterpret_cast<f32x4 *>(dst + i) =
                    f32x4{o[s][2 * k][i >> 1], o[s][2 * k + 1][i >> 1], o[s][2 * k][(i >> 1) + 1],
                          o[s][2 * k + 1][(i >> 1) + 1]} * f;
        }
    }
    __syncthreads();
    for (int e = tid; e < hp * kCols * DB * 4; e += kAttnWaves * 64) {
        const int ch = (e % (DB * 4)) * 8, col = (e / (DB * 4)) % kCols, w = e / (DB * 4 * kCols);
        float mx = -kInf, sum = 0.0f, x[8] = {};
        for (int p = 0; p < parts; ++p) mx = fmaxf(mx, ml[(p * hp + w) * kCols + col][0]);
        for (int p = 0; p < parts; ++p) {
            const f32x2 v = ml[(p * hp + w) * kCols + col];
            sum += v[1] * __builtin_amdgcn_exp2f(v[0] - (mx == -kInf ? 0.0f : mx));
            const float *src = acc + ((p * hp + w) * kCols + col) * (kDP + 4) + ch;
#pragma unroll
            for (int i = 0; i < 8; ++i) x[i] += src[i];
        }
        finish(col, h0 + w, ch, mx, sum, x);
    }
}

// Columns of one workgroup: 32 queries, or 16 where there are no more and for heads of more
// than 64 channels, whose sums would fill the registers.
template <typename T, int DB, int NS, bool PAGED, int TERMS>
void run_fwd(const AttnArgs &a, hipStream_t s) {
    const dim3 grid(xcd_grid(a.nwg, a.per)), block(kAttnWaves * 64);
    const FwdLds lds = fwd_lds(16 * NS, 32 * DB, a.hp, a.parts, a.rule.nb, a.bias != nullptr);
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
