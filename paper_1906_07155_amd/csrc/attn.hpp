// attn.hpp -- device-side parts shared by the attention kernels of the relation head.
//
// Every product runs on 16x16 matrix instructions.  Operand layouts (lane l, n = l % 16,
// g = l / 16): A holds row n, B holds column n, both the k-slots 8g .. 8g + 7 of a step of
// 32; the result has column n and rows 4g + i, i = 0..3.  Binary32 has steps of 4, k-slot g:
// eight of them, the j-th taking element j of the same registers, make the same step of 32.
//
// Three things follow from the freedom to order rows and k-slots as one likes:
//   - Row r of the first of two 16-row tiles is streamed row 8 (r / 4) + r % 4, of the second
//     four rows further on.  A lane's results, rows 4g + i of either, are then streamed rows
//     8g .. 8g + 7 in order, and as they stand its B operand of a step of 32: the softmax
//     weights never leave their lane, and masks, scales and buckets of a lane's eight rows
//     are adjacent in memory.
//   - The transposed operand (channels as rows, streamed rows as k-slots) of bf16 data is
//     read from LDS, where a tile's rows are put by loads that go there directly: the
//     transposing read gives a lane one channel of four rows.  (Read from memory as pairs
//     of channels a tile of 64 channels takes 16 loads of 4 bytes a lane instead of 4 of 16,
//     and each costs the address unit the same 16 cycles.  16 images of up to 1000 boxes in 16
//     heads of 64 channels, weights in one part: forward 197 us that way, 173 this way.)
//   - Binary32 data has no such read: lane n takes channels 2n and 2n + 1 of its eight
//     rows from memory, the operands of two tiles with channel 2r + t in row r of tile t.
#pragma once

#include "relation.hpp"

namespace rex {

using f32x4 = float __attribute__((ext_vector_type(4)));
using f32x2 = float __attribute__((ext_vector_type(2)));
using f32x8 = float __attribute__((ext_vector_type(8)));
using bf16x8 = __bf16 __attribute__((ext_vector_type(8)));
using i32x4 = int __attribute__((ext_vector_type(4)));

constexpr float kInf = __builtin_inff();

template <typename T> struct Num;     // the operands of one type

template <> struct Num<uint16_t> {    // bf16
    using Frag = bf16x8;
    using Pair = uint32_t;            // two adjacent channels
    static constexpr int kSize = 2;
    static __device__ __forceinline__ Frag zero() { return Frag{}; }
    static __device__ __forceinline__ Frag load(const char *p) {
        return *(const REX_GLOBAL Frag *)(p);
    }
    static __device__ __forceinline__ Frag load(__amdgpu_buffer_rsrc_t r, uint32_t off, uint32_t soff) {
        return __builtin_bit_cast(Frag, __builtin_amdgcn_raw_buffer_load_b128(r, off, soff, 0));
    }
    static __device__ __forceinline__ Pair load_pair(__amdgpu_buffer_rsrc_t r, uint32_t off, uint32_t soff) {
        return __builtin_amdgcn_raw_buffer_load_b32(r, off, soff, 0);
    }
    static __device__ __forceinline__ f32x4 mma(Frag a, Frag b, f32x4 c) {
        return __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, b, c, 0, 0, 0);
    }
    // the two 16-channel operands of eight pairs
    static __device__ __forceinline__ void split(const Pair (&x)[8], Frag &lo, Frag &hi) {
        u32x4 a, b;
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            a[j] = __builtin_amdgcn_perm(x[2 * j + 1], x[2 * j], 0x05040100u);
            b[j] = __builtin_amdgcn_perm(x[2 * j + 1], x[2 * j], 0x07060302u);
        }
        lo = __builtin_bit_cast(Frag, a);
        hi = __builtin_bit_cast(Frag, b);
    }
    static __device__ __forceinline__ Frag round(const float (&x)[8]) {
        Frag f;
#pragma unroll
        for (int j = 0; j < 8; ++j) f[j] = static_cast<__bf16>(x[j]);
        return f;
    }
    static constexpr bool kExact = false;     // round() rounds
    // x cut to bf16 (toward zero: one operation, and the rest is exact), and x left with what
    // that cut off
    static __device__ __forceinline__ Frag cut_off(float (&x)[8]) {
        u32x4 f;
#pragma unroll
        for (int j = 0; j < 4; ++j)
            f[j] = __builtin_amdgcn_perm(__float_as_uint(x[2 * j + 1]), __float_as_uint(x[2 * j]), 0x07060302u);
#pragma unroll
        for (int j = 0; j < 8; ++j) x[j] -= __uint_as_float(__float_as_uint(x[j]) & 0xffff0000u);
        return __builtin_bit_cast(Frag, f);
    }
    // eight channels to memory
    static __device__ __forceinline__ void store(char *p, const float (&x)[8]) {
        *(REX_GLOBAL Frag *)(p) = round(x);
    }
    static __device__ __forceinline__ void store4(char *p, f32x4 x) {
        using bf16x4 = __bf16 __attribute__((ext_vector_type(4)));
        *(REX_GLOBAL bf16x4 *)(p) = bf16x4{static_cast<__bf16>(x[0]), static_cast<__bf16>(x[1]),
                                           static_cast<__bf16>(x[2]), static_cast<__bf16>(x[3])};
    }
    // keeps the elements whose bit of m is set
    static __device__ __forceinline__ void keep(Frag &f, uint32_t m) {
        u32x4 v = __builtin_bit_cast(u32x4, f);
#pragma unroll
        for (int j = 0; j < 4; ++j)
            v[j] &= (m >> (2 * j) & 1u ? 0xffffu : 0u) | (m >> (2 * j + 1) & 1u ? 0xffff0000u : 0u);
        f = __builtin_bit_cast(Frag, v);
    }
    // four codes of the memory -> four numbers
    static __device__ __forceinline__ void widen(Frag &f, int at, uint32_t c) {
#pragma unroll
        for (int j = 0; j < 4; ++j)
            f[at + j] = static_cast<__bf16>(static_cast<float>(static_cast<int8_t>(c >> (8 * j))));
    }
};

template <> struct Num<float> {
    using Frag = f32x8;
    using Pair = f32x2;
    static constexpr int kSize = 4;
    static __device__ __forceinline__ Frag zero() { return Frag{}; }
    static __device__ __forceinline__ Frag load(const char *p) {
        const f32x4 a = *(const REX_GLOBAL f32x4 *)(p);
        const f32x4 b = *(const REX_GLOBAL f32x4 *)(p + 16);
        return Frag{a[0], a[1], a[2], a[3], b[0], b[1], b[2], b[3]};
    }
    static __device__ __forceinline__ Frag load(__amdgpu_buffer_rsrc_t r, uint32_t off, uint32_t soff) {
        const f32x4 a = __builtin_bit_cast(f32x4, __builtin_amdgcn_raw_buffer_load_b128(r, off, soff, 0));
        const f32x4 b = __builtin_bit_cast(f32x4, __builtin_amdgcn_raw_buffer_load_b128(r, off + 16, soff, 0));
        return Frag{a[0], a[1], a[2], a[3], b[0], b[1], b[2], b[3]};
    }
    static __device__ __forceinline__ Pair load_pair(__amdgpu_buffer_rsrc_t r, uint32_t off, uint32_t soff) {
        return __builtin_bit_cast(f32x2, __builtin_amdgcn_raw_buffer_load_b64(r, off, soff, 0));
    }
    static __device__ __forceinline__ f32x4 mma(Frag a, Frag b, f32x4 c) {
#pragma unroll
        for (int j = 0; j < 8; ++j) c = __builtin_amdgcn_mfma_f32_16x16x4f32(a[j], b[j], c, 0, 0, 0);
        return c;
    }
    static __device__ __forceinline__ void split(const Pair (&x)[8], Frag &lo, Frag &hi) {
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            lo[j] = x[j][0];
            hi[j] = x[j][1];
        }
    }
    static __device__ __forceinline__ Frag round(const float (&x)[8]) {
        return Frag{x[0], x[1], x[2], x[3], x[4], x[5], x[6], x[7]};
    }
    static constexpr bool kExact = true;
    static __device__ __forceinline__ Frag cut_off(float (&x)[8]) { return round(x); }
    static __device__ __forceinline__ void store(char *p, const float (&x)[8]) {
        *(REX_GLOBAL f32x4 *)(p) = f32x4{x[0], x[1], x[2], x[3]};
        *(REX_GLOBAL f32x4 *)(p + 16) = f32x4{x[4], x[5], x[6], x[7]};
    }
    static __device__ __forceinline__ void store4(char *p, f32x4 x) { *(REX_GLOBAL f32x4 *)(p) = x; }
    static __device__ __forceinline__ void keep(Frag &f, uint32_t m) {
#pragma unroll
        for (int j = 0; j < 8; ++j) f[j] = m >> j & 1u ? f[j] : 0.0f;
    }
    static __device__ __forceinline__ void widen(Frag &f, int at, uint32_t c) {
#pragma unroll
        for (int j = 0; j < 4; ++j) f[at + j] = static_cast<float>(static_cast<int8_t>(c >> (8 * j)));
    }
};

// acc += A x for weights x of which bf16 takes the first TERMS parts of eight bits: 2 leaves up to
// 2^-17 of them out, far below what rounding a bf16 result does, and 3 nothing.  (One part, that is
// weights rounded to bf16, would add as much error as the result's own rounding: 2.3e-3 of the results'
// norm instead of 1.7e-3.  16 images of up to 1000 boxes in 16 heads of 64 channels: forward 181 us
// with one part, 210 with two, 232 with three; backward 700 and 756.)
template <typename T, int TERMS, int NT>
__device__ __forceinline__ void add_weighted(const typename Num<T>::Frag (&rows)[NT], float (&x)[8],
                                             f32x4 (&acc)[NT]) {
    using N = Num<T>;
#pragma unroll
    for (int i = 0; i < (N::kExact ? 1 : TERMS); ++i) {
        const typename N::Frag f = i + 1 < TERMS ? N::cut_off(x) : N::round(x);
#pragma unroll
        for (int k = 0; k < NT; ++k) acc[k] = N::mma(rows[k], f, acc[k]);
    }
}

// The first `rows` rows of one head of one image, read through a buffer resource that starts
// at a tile's first row: a lane's 32-bit offset past the last row (or marked kBufOOB:
// channels past D) reads 0 without an access, so tiles may run over the end and padding is
// never read, and the lane offsets are the same for every tile.  The host checks that
// (rows + 32) * stride stays below kBufMaxBytes, so no offset wraps.
struct HeadRows {
    const char *base;
    uint32_t bytes, sr;       // bytes that may be read; from row to row
    __device__ __forceinline__ __amdgpu_buffer_rsrc_t at(int row) const {   // row < rows, uniform
        const uint32_t skip = static_cast<uint32_t>(row) * sr;
        return make_rsrc(base + skip, bytes - skip);
    }
};
template <typename T>
__device__ __forceinline__ HeadRows head_rows(const Rows &x, int b, int head, int rows, int D) {
    const char *base = static_cast<const char *>(x.p) + b * x.sb + static_cast<int64_t>(head) * x.sh;
    const uint32_t bytes = rows > 0 ? static_cast<uint32_t>(rows - 1) * x.sr + D * Num<T>::kSize : 0u;
    return HeadRows{base, bytes, x.sr};
}
// Lane offsets in a tile of 32 streamed rows.  f: of the operand whose rows are rows (see the
// top of this file), channels 32k + 8g ..; p: of the one whose rows are channels, 32k + 2n
// and the next, of the rows 8g + j.
template <typename T, int DB>
struct TileOffsets {
    using N = Num<T>;
    uint32_t f[DB], p[DB], sr;
    __device__ __forceinline__ TileOffsets(uint32_t sr_, int n, int g, int D) : sr(sr_) {
#pragma unroll
        for (int k = 0; k < DB; ++k) {
            f[k] = 32 * k + 8 * g < D ? (8 * (n >> 2) + (n & 3)) * sr + (32 * k + 8 * g) * N::kSize : kBufOOB;
            p[k] = 32 * k + 2 * n < D ? 8 * g * sr + (32 * k + 2 * n) * N::kSize : kBufOOB;
        }
    }
    // The rows' offsets go through the scalar register of the load where all 32 rows are there:
    // the range check does not see it, and no lane register is needed for it.
    __device__ __forceinline__ void frags(__amdgpu_buffer_rsrc_t r, bool inside, typename N::Frag (&x)[2][DB]) const {
        if (inside) {
#pragma unroll
            for (int t = 0; t < 2; ++t)
#pragma unroll
                for (int k = 0; k < DB; ++k) x[t][k] = N::load(r, f[k], 4 * t * sr);
        } else {
#pragma unroll
            for (int t = 0; t < 2; ++t)
#pragma unroll
                for (int k = 0; k < DB; ++k) x[t][k] = N::load(r, f[k] + 4 * t * sr, 0);
        }
    }
    __device__ __forceinline__ void pairs(__amdgpu_buffer_rsrc_t r, bool inside, typename N::Pair (&x)[DB][8]) const {
        if (inside) {
#pragma unroll
            for (int j = 0; j < 8; ++j)
#pragma unroll
                for (int k = 0; k < DB; ++k) x[k][j] = N::load_pair(r, p[k], j * sr);
        } else {
#pragma unroll
            for (int j = 0; j < 8; ++j)
#pragma unroll
                for (int k = 0; k < DB; ++k) x[k][j] = N::load_pair(r, p[k] + j * sr, 0);
        }
    }
};
// Column operands: rows 16 s + n from the resource's first row on.
template <typename T, int DB, int NS>
__device__ __forceinline__ void load_columns(__amdgpu_buffer_rsrc_t r, uint32_t sr, int n, int g, int D,
                                             typename Num<T>::Frag (&x)[NS][DB]) {
#pragma unroll
    for (int s = 0; s < NS; ++s)
#pragma unroll
        for (int k = 0; k < DB; ++k) {
            const int ch = 32 * k + 8 * g;
            x[s][k] = Num<T>::load(r, ch < D ? (16 * s + n) * sr + ch * Num<T>::kSize : kBufOOB, 0);
        }
}

// One wave's tile of 32 bf16 rows in LDS, 64 * DB bytes a row, and its two readings.  Loads
// put 16 bytes of each lane at consecutive places, so which chunk of a row a lane loads is
// what spreads the reads over the banks: chunk c of row r is at place c ^ f(r), f chosen
// such that the 32 lanes of half a transposing read (rows 0-3 and 8-11 of some eight-row
// blocks) meet 32 different pairs of banks.  What lies past the resource's end is zeros.
// (the host's pass over kernels knows neither LDS nor these loads)
#ifdef __HIP_DEVICE_COMPILE__
#define REX_LDS __attribute__((address_space(3)))
#else
#define REX_LDS
#endif
template <int DB>
struct LdsTile {
    using Place = REX_LDS char *;
    static constexpr int kBytes = kTile * 64 * DB, kChunks = 4 * DB, kRows = 16 / DB;   // rows of one load
    Place at;                         // the wave's tile, or the first of several one after the other
    Place nat[DB], tr[2 * DB];        // a lane's places in the two readings
    static __device__ __forceinline__ int turn(int r) {
        return 2 * (((r & 3) | (r >> 1 & 4)) >> (DB == 1 ? 2 : DB == 2 ? 1 : 0));
    }
    __device__ __forceinline__ LdsTile(char *at_, int lane) : at((Place)at_) {
        const int n = lane & 15, g = lane >> 4;
        // four rows on, r & 3 and r >> 3 and so the turn are the same: a constant offset
        const int r = 8 * (n >> 2) + (n & 3), q = 8 * g + (n >> 2);
#pragma unroll
        for (int k = 0; k < DB; ++k) nat[k] = at + r * 64 * DB + ((4 * k + g) ^ turn(r)) * 16;
#pragma unroll
        for (int u = 0; u < 2 * DB; ++u)
            tr[u] = at + q * 64 * DB + ((2 * u + (n >> 1 & 1)) ^ turn(q)) * 16 + (n & 1) * 8;
    }
    // Lane offsets of the loads of even- and odd-numbered eight-row blocks.
    struct Loads {
        uint32_t off[2], sr;
        __device__ __forceinline__ Loads(uint32_t sr_, int lane, int D) : sr(sr_) {
            const int row = lane / kChunks;
#pragma unroll
            for (int e = 0; e < 2; ++e) {
                const int chunk = (lane % kChunks) ^ turn(row + (DB == 1 ? 0 : 8 * e));
                off[e] = 8 * chunk < D ? row * sr + chunk * 16 : kBufOOB;
            }
        }
    };
    // Every reading of the last tile has to be back before the next is on its way (a load to LDS
    // is not ordered with the wave's LDS reads), and a tile has to be there before it is read.
    static __device__ __forceinline__ void released() { asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory"); }
    static __device__ __forceinline__ void arrived() { asm volatile("s_waitcnt vmcnt(0)" ::: "memory"); }
    __device__ __forceinline__ void fill(__amdgpu_buffer_rsrc_t r, bool inside, const Loads &l, int which = 0) const {
#ifdef __HIP_DEVICE_COMPILE__
#pragma unroll
        for (int i = 0; i < 2 * DB; ++i) {
            const int odd = DB == 4 ? i >> 1 & 1 : DB == 2 ? i & 1 : 0;
            auto *to = (REX_LDS void *)(at + which * kBytes + i * 1024);
            if (inside) __builtin_amdgcn_raw_ptr_buffer_load_lds(r, to, 16, l.off[odd], i * kRows * l.sr, 0, 0);
            else __builtin_amdgcn_raw_ptr_buffer_load_lds(r, to, 16, l.off[odd] + i * kRows * l.sr, 0, 0, 0);
        }
#endif
    }
    // the operand whose rows are rows: tile t, channels 32k + 8g ..
    __device__ __forceinline__ bf16x8 rows(int t, int k, int which = 0) const {
        return *(const REX_LDS bf16x8 *)(nat[k] + which * kBytes + 4 * t * 64 * DB);
    }
    // the operand whose rows are channels: tile u, channel 16u + n
    __device__ __forceinline__ bf16x8 channels(int u, int which = 0) const {
#ifdef __HIP_DEVICE_COMPILE__
        using s16x4 = short __attribute__((ext_vector_type(4)));
        using s16x8 = short __attribute__((ext_vector_type(8)));
        s16x4 x[2];
#pragma unroll
        for (int e = 0; e < 2; ++e)
            x[e] = __builtin_amdgcn_ds_read_tr16_b64_v4i16(
                (REX_LDS s16x4 *)(tr[u] + which * kBytes + 4 * e * 64 * DB));
        return __builtin_bit_cast(bf16x8, s16x8{x[0][0], x[0][1], x[0][2], x[0][3], x[1][0], x[1][1], x[1][2], x[1][3]});
#else
        return bf16x8{};
#endif
    }
};

// Largest / sum over the four lanes that share a column (l, l ^ 16, l ^ 32, l ^ 48).
__device__ __forceinline__ float max_over_rows(float x) {
    x = fmaxf(x, __shfl_xor(x, 16));
    return fmaxf(x, __shfl_xor(x, 32));
}
__device__ __forceinline__ float sum_over_rows(float x) {
    x += __shfl_xor(x, 16);
    return x + __shfl_xor(x, 32);
}

// The four adjacent channels that quad u of a lane's results (2 * DB tiles of 16 channels) are,
// and their values.  NATURAL: channels in the tiles' order, else interleaved by pairs.
template <bool NATURAL>
__device__ __forceinline__ int quad_channel(int u, int g) {
    return NATURAL ? 16 * u + 4 * g : 32 * (u >> 1) + 8 * g + 4 * (u & 1);
}
template <bool NATURAL, int NT>
__device__ __forceinline__ f32x4 quad_values(const f32x4 (&o)[NT], int u) {
    if constexpr (NATURAL) return o[u];
    const int k = u & ~1, i = 2 * (u & 1);
    return f32x4{o[k][i], o[k + 1][i], o[k][i + 1], o[k + 1][i + 1]};
}

// A box as the bucket rule sees it: centre and, for a query, 1 / side.
struct BoxGeo {
    float cx, cy, ix, iy;
};
__device__ __forceinline__ f32x4 box_load(const float *p) {
    gcptr<float> b = as_global<float>(p);
    return f32x4{b[0], b[1], b[2], b[3]};
}
__device__ __forceinline__ void box_centre(f32x4 b, float &cx, float &cy) {
    cx = (b[0] + b[2]) * 0.5f;
    cy = (b[1] + b[3]) * 0.5f;
}
__device__ __forceinline__ BoxGeo box_geo(f32x4 b) {
    BoxGeo o;
    box_centre(b, o.cx, o.cy);
    o.ix = 1.0f / fmaxf(b[2] - b[0], 1.0f);
    o.iy = 1.0f / fmaxf(b[3] - b[1], 1.0f);
    return o;
}
// Bucket of one axis, 0 .. 2 * half.  The magnitude's edges are binary32 numbers whose low
// bits are 0, so counting those reached is a shift of the bits of |r|.
__device__ __forceinline__ int axis_bucket(float r, const BucketRule &b) {
    const int e = static_cast<int>(__builtin_amdgcn_ubfe(__float_as_uint(r), b.shift, 31 - b.shift));
    const int m = min(max(e, b.base - 1), b.base - 1 + b.half);        // edges reached + base - 1
    return r < 0.0f ? b.half + b.base - 1 - m : m + (b.half - b.base + 1);
}
// Byte offset of a pair's entry in one head's table.
__device__ __forceinline__ uint32_t pair_bucket(const BoxGeo &q, float kx, float ky,
                                                const BucketRule &b) {
    const uint32_t bx = axis_bucket((kx - q.cx) * q.ix, b);
    const uint32_t by = axis_bucket((ky - q.cy) * q.iy, b);
    return __umul24(by, 4 * b.nb) + 4 * bx;
}

// An entry of a head's table in LDS, so that it can be what a logit's sum starts with: in
// units of the plain products (divided by the scale; what that takes past the finite numbers stays
// finite).  Masks written as a type's lowest value count as -inf.
constexpr float kLowest = -1e30f;
__device__ __forceinline__ float table_entry(float bias, float scale) {
    const float x = bias / scale;
    return bias <= kLowest ? -kInf : fabsf(x) == kInf ? copysignf(3.4028234664e38f, x) : x;
}
// A table with a large entry (a mask of -1e9, say) is not used so: a row all of whose keys are at
// such an entry needs the differences of its entries and of its products, which the entry would
// drown.  Its sums start from (entry - offset) / scale, the offset being the row's largest entry, and
// the entries are those in memory.  (Branches for that cost the other calls some 5 %: forward of 1000
// boxes in 16 heads of 64 channels 26.2 us without them, 27.3 with; loops of its own in the same
// kernels cost more, by the registers of both.)
constexpr float kWideBias = 64.0f;
__device__ __forceinline__ bool wide_table(const char *tab, int n, float scale, int lane) {
    bool wide = false;
#pragma unroll 4
    for (int i = lane; i < n; i += 64) {
        const float x = reinterpret_cast<const float *>(tab)[i];
        wide |= x != -kInf && fabsf(x) * scale > kWideBias;
    }
    return __any(wide);
}

// The table entries of a lane's eight rows: `at` holds 16-bit byte offsets into the head's
// table in LDS.
__device__ __forceinline__ uint32_t table_offset(u32x4 at, int j) {
    return j & 1 ? at[j >> 1] >> 16 : at[j >> 1] & 0xffffu;
}
__device__ __forceinline__ void table_gather(u32x4 at, const char *tab, f32x4 (&x)[2]) {
#pragma unroll
    for (int j = 0; j < 8; ++j)
        x[j >> 2][j & 3] = *reinterpret_cast<const float *>(tab + table_offset(at, j));
}
// The same of a table in memory, natural units.
__device__ __forceinline__ float wide_entry(const float *bias, uint32_t offset) {
    const float x = as_global<float>(bias)[offset / 4];
    return x <= kLowest ? -kInf : x;
}
__device__ __forceinline__ void wide_gather(u32x4 at, const float *bias, f32x4 (&x)[2]) {
#pragma unroll
    for (int j = 0; j < 8; ++j) x[j >> 2][j & 3] = wide_entry(bias, table_offset(at, j));
}

constexpr int kBuckStride = 40;   // 16-bit entries of one column's 32 rows in LDS (16-byte reads
                                  // of 16 columns then spread over the banks)

// Workgroups go to the eight XCDs in turn.  `per` workgroups that share keys (one image and
// head group) belong on one XCD, whose L2 then holds those keys: such sets go to the XCDs in
// turn where there are enough of them to spread the images' different lengths (16 ragged
// images, 2 head groups: forward 1.25 times faster than runs of neighbouring images), else
// each XCD gets a run of neighbouring workgroups.  The grid is `xcd_grid(sets * per, per)`.
inline __host__ __device__ bool xcd_sets(int sets) { return sets >= 64 || (sets >= 8 && sets % 8 == 0); }
inline __host__ __device__ int xcd_grid(int n, int per) {
    const int sets = n / per;
    return xcd_sets(sets) ? (sets + 7) / 8 * 8 * per : (n + 7) & ~7;
}
// Workgroup id -> [0, n), or n and more for those that are left over.
__device__ __forceinline__ int xcd_order(int id, int n, int per) {
    const int xcd = id & 7, slot = id >> 3;
    if (xcd_sets(n / per)) return (xcd + 8 * (slot / per)) * per + slot % per;
    return xcd * ((n + 7) >> 3) + slot;
}

}  // namespace rex
