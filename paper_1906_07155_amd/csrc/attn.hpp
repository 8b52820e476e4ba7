// attn.hpp -- device-side parts shared by the attention kernels of the relation head.
//
// Every product runs on 16x16 matrix instructions.  Operand layouts (lane l, n = l % 16,
// g = l / 16): A holds row n, B holds column n, both the k-slots 8g .. 8g + 7 of a step of
// 32; the result has column n and rows 4g + i, i = 0..3.  Binary32 has steps of 4, k-slot g:
// eight of them, the j-th taking element j of the same registers, make the same step of 32.
//
// Two things follow from the freedom to order rows and k-slots as one likes:
//   - A lane's results of two 16-row tiles (rows 4g + i of either) are, as they stand, its B
//     operand of a step of 32 in which slot 8g + j is row 4g + j of the first tile (j < 4)
//     or row 4g + j - 4 of the second: the softmax weights never leave their lane.
//   - The transposed operand (channels as rows) is read straight from row-major memory: lane
//     n takes channels 2n and 2n + 1 of its eight rows, and the low and the high halves
//     are the A operands of two 16-channel tiles, channel 2r + t in row r of tile t.  Of the
//     two results a lane then holds channels 8g .. 8g + 7 of its column: one 16-byte store.
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
    static __device__ __forceinline__ Pair no_pair() { return 0u; }
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
    static constexpr bool kExact = false;     // round() cuts off
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
    static __device__ __forceinline__ Pair no_pair() { return Pair{}; }
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
    static __device__ __forceinline__ void widen(Frag &f, int at, uint32_t c) {
#pragma unroll
        for (int j = 0; j < 4; ++j) f[at + j] = static_cast<float>(static_cast<int8_t>(c >> (8 * j)));
    }
};

// acc += A x for weights x of which bf16 takes the first TERMS parts of eight bits: 1 rounds
// them, 2 leaves up to 2^-16 of them out, 3 nothing.
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
// Lane offsets in a tile of 32 rows.  f: of the operand whose rows are rows (n and 16 + n,
// channels 32k + 8g ..); p: of the one whose rows are channels (32k + 2n and the next, of
// the rows slot_row(g, j)).
template <typename T, int DB>
struct TileOffsets {
    uint32_t f[DB], p[DB], sr;
    __device__ __forceinline__ TileOffsets(uint32_t sr_, int n, int g, int D) : sr(sr_) {
#pragma unroll
        for (int k = 0; k < DB; ++k) {
            f[k] = 32 * k + 8 * g < D ? n * sr + (32 * k + 8 * g) * Num<T>::kSize : kBufOOB;
            p[k] = 32 * k + 2 * n < D ? 4 * g * sr + (32 * k + 2 * n) * Num<T>::kSize : kBufOOB;
        }
    }
    // The rows' offsets go through the scalar register of the load where all 32 rows are there:
    // the range check does not see it, and no lane register is needed for it.
    __device__ __forceinline__ void frags(__amdgpu_buffer_rsrc_t r, bool inside,
                                          typename Num<T>::Frag (&x)[2][DB]) const {
        if (inside) {
#pragma unroll
            for (int t = 0; t < 2; ++t)
#pragma unroll
                for (int k = 0; k < DB; ++k) x[t][k] = Num<T>::load(r, f[k], 16 * t * sr);
        } else {
#pragma unroll
            for (int t = 0; t < 2; ++t)
#pragma unroll
                for (int k = 0; k < DB; ++k) x[t][k] = Num<T>::load(r, f[k] + 16 * t * sr, 0);
        }
    }
    __device__ __forceinline__ void pairs(__amdgpu_buffer_rsrc_t r, bool inside,
                                          typename Num<T>::Pair (&x)[DB][8]) const {
        if (inside) {
#pragma unroll
            for (int j = 0; j < 8; ++j)
#pragma unroll
                for (int k = 0; k < DB; ++k) x[k][j] = Num<T>::load_pair(r, p[k], (j < 4 ? j : 12 + j) * sr);
        } else {
#pragma unroll
            for (int j = 0; j < 8; ++j)
#pragma unroll
                for (int k = 0; k < DB; ++k) x[k][j] = Num<T>::load_pair(r, p[k] + (j < 4 ? j : 12 + j) * sr, 0);
        }
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

// Row of the streamed 32 that element j of a lane's operand is (see above).
__device__ __forceinline__ int slot_row(int g, int j) { return j < 4 ? 4 * g + j : 12 + 4 * g + j; }

// A box as the bucket rule sees it: centre and, for a query, 1 / side.
struct BoxGeo {
    float cx, cy, ix, iy;
};
__device__ __forceinline__ void box_centre(const REX_GLOBAL float *b, float &cx, float &cy) {
    cx = (b[0] + b[2]) * 0.5f;
    cy = (b[1] + b[3]) * 0.5f;
}
__device__ __forceinline__ BoxGeo box_geo(const REX_GLOBAL float *b) {
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
// units of the plain products (divided by the scale).  Masks written as a type's lowest
// value count as -inf: kept as numbers they would drown the logits they are added to.
__device__ __forceinline__ float table_entry(float bias, float scale) {
    return bias <= -1e30f ? -kInf : bias / scale;
}

// The table entries of a lane's four rows: `at` holds four 16-bit byte offsets, `tab` (an LDS
// address below 2^16) the head's table.
__device__ __forceinline__ f32x4 table_gather(u32x2 at, const char *tab) {
    f32x4 v;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const uint32_t off = i & 1 ? at[i >> 1] >> 16 : at[i >> 1] & 0xffffu;
        v[i] = *reinterpret_cast<const float *>(tab + off);
    }
    return v;
}

constexpr int kBuckStride = 36;   // 16-bit entries of one column's 32 rows in LDS (8-byte reads
                                  // of 16 columns then start in 16 different bank pairs)

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
