// gemm.hpp -- tiled products of the dense layers, out[m][n] = sum_k Q(m, k) P(n, k).
//
// A workgroup owns BM x BN results; both operands' tiles of 128 bytes of k (64 bf16, 32 binary32)
// go to LDS by loads that write there directly, the next step's into a second buffer while this
// step's products run.  P's rows are the rows of the 16x16 products and Q's their columns, so a
// lane's four results of one product are adjacent in the output's row.
//
// Operands lie in memory with k adjacent, or transposed with their rows adjacent (the gradients'
// products).  16-byte chunks of a tile's rows are spread over the banks by an exclusive or of the
// chunk's number with bits of the row's (chosen on the loading side: a lane's load goes to a fixed
// place, and which chunk it fetches is free):
//   k adjacent: [row][k], 8 chunks a row; a lane reads a chunk of its row.  Rows are ordered as in
//     attn.hpp, so that two products' rows are eight adjacent results of a lane.
//   transposed: [k][row]; bf16 goes through the transposing read, binary32 reads four k one by one
//     (its products take 32 cycles each: reading is no bound).
//
// Nothing outside an operand is used: chunks past the last row, and past the last k of the last
// step, are given an offset that the range check answers with 0.
//
// What bounds it: bf16, the products and what feeds them, which take turns at a step's barrier (one
// workgroup of eight waves on a CU, of 128 x 64 results each: 8192^3 852 to 875 us, 1.26 to 1.29 PFLOP/s, where
// a library's product takes 800; tiles of 128 x 128 1045, 64 x 64 1590), and around the loop the epilogue, which
// nothing of the same CU hides: 16000 x 2048 x 1024 with gelu and its slopes 109 us, of which the matrix
// instructions take 29 % and the vector instructions 51 (16000 x 1024 x 2048 without either 70, 47 % and 25).
// Lines of 64 bytes of k in three or four buffers, four waves of 128 x 128, operands read half a step ahead
// and raised priorities of waves were no faster.
// binary32, the products: 83 % of the time of 1024 x 12544 x 1024 (three tiles of 128 x 64 on a CU, those of the
// last round in parts: 237 us, 111 TFLOP/s; 4096^3 1020 us, 135).
#pragma once

#include "epilogue.hpp"

namespace rex {

#ifdef __HIP_DEVICE_COMPILE__
#define REX_LDS_LOAD(r, to, off) __builtin_amdgcn_raw_ptr_buffer_load_lds(r, (REX_LDS void *)(to), 16, off, 0, 0, 0)
#else
#define REX_LDS_LOAD(r, to, off) (void)0
#endif

// The products of a type: 16 x 16 results, rows 4g .. 4g + 3 (g = l / 16) of column l % 16 in lane l.
// (32x32x16 products of bf16 read half as many operands' registers, and yet 8192^3 took 1030 us with
// them where it took 935 on the same card.)
template <typename T> struct Shape;
template <> struct Shape<uint16_t> {
    using Frag = bf16x8;
    static constexpr int kParts = 1;
    static __device__ __forceinline__ f32x4 mma(Frag a, Frag b, f32x4 c, int) {
        return __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, b, c, 0, 0, 0);
    }
};
template <> struct Shape<float> {
    using Frag = f32x4;
    static constexpr int kParts = 4;         // of an operand's registers, one product each
    static __device__ __forceinline__ f32x4 mma(Frag a, Frag b, f32x4 c, int part) {
        return __builtin_amdgcn_mfma_f32_16x16x4f32(a[part], b[part], c, 0, 0, 0);
    }
};

// One operand's tile of ROWS rows, 128 bytes of k each.
template <typename T, bool TR, int ROWS, int WAVES, bool WHOLE>
struct Side {
    static constexpr int kSize = sizeof(T), kChunk = 16 / kSize, kStep = 128 / kSize;   // elements
    static constexpr int kBytes = ROWS * 128, kLoads = kBytes / (1024 * WAVES);         // of a wave
    static constexpr int kPitch = TR ? ROWS * kSize : 128, kPieces = kPitch / 16;       // of a line
    using Frag = typename Shape<T>::Frag;
    using Place = REX_LDS char *;

    // what the loads need: the lane's offsets, and the k and first row of its chunks in a step
    const char *origin;
    int64_t step_bytes;
    uint32_t off[kLoads];
    int k[kLoads], e[WHOLE ? 1 : kLoads];
    int left_k, left_rows;
    u32x4 held[2][WHOLE ? 1 : kLoads];        // of this step and the next

    // What spreads a line's chunks over the banks for the lanes that read together: eight lanes with a
    // chunk of eight rows each (k adjacent); 32 lanes with 32 bytes of eight lines (transposed bf16: lines
    // 0-3 and 8-11 of 16), 64 with 64 bytes of every fourth line (transposed binary32).
    static __device__ __forceinline__ int turn(int line) {
        if (!TR) return line & 7;
        if (kSize == 4) return 4 * (line >> 2 & 3);
        return 2 * (((line & 3) | (line >> 1 & 4)) >> (ROWS == 64 ? 1 : 0));
    }

    __device__ __forceinline__ Side(const void *p, int64_t ld, int row0, int rows, int k0, int K, int wave, int lane) {
        origin = static_cast<const char *>(p) + (TR ? k0 * ld + static_cast<int64_t>(row0) * kSize
                                                    : row0 * ld + static_cast<int64_t>(k0) * kSize);
        step_bytes = TR ? kStep * ld : kStep * kSize;
        left_k = K - k0;
        left_rows = rows - row0;
#pragma unroll
        for (int i = 0; i < kLoads; ++i) {
            const int j = (i * WAVES + wave) * 64 + lane, line = j / kPieces;
            const int chunk = (j % kPieces) ^ turn(line);
            off[i] = static_cast<uint32_t>(line * ld) + chunk * 16;
            k[i] = TR ? line : chunk * kChunk;
            const int row = TR ? chunk * kChunk : line;
            if (WHOLE && row >= left_rows) off[i] = kBufOOB;
            if (!WHOLE) e[i] = row;
        }
    }

    // the next tile on its way to `to` (WHOLE), or to registers
    __device__ __forceinline__ void load(char *to, int wave, int which = 0) {
        if constexpr (WHOLE) {
            const auto r = make_rsrc(origin, kBufMaxBytes - 1);
            const bool all = left_k >= kStep;
#pragma unroll
            for (int i = 0; i < kLoads; ++i)
                REX_LDS_LOAD(r, to + (i * WAVES + wave) * 1024, all || k[i] < left_k ? off[i] : kBufOOB);
        } else if (kSize == 4 && left_k >= kStep && left_rows >= ROWS) {
            // nothing of the tile is outside (4096 x 4097 x 4095: 1312 -> 1167 us; of bf16, whose eight elements
            // beside it stay in the same loop, 237 -> 248)
            using Any = uint32_t __attribute__((ext_vector_type(4), aligned(sizeof(T))));
#pragma unroll
            for (int i = 0; i < kLoads; ++i) held[which][i] = *(const REX_GLOBAL Any *)(origin + off[i]);
        } else {
#pragma unroll
            for (int i = 0; i < kLoads; ++i) {
                // a chunk at any address where all of it is there, else its elements
                const int there = TR ? left_rows - e[i] : left_k - k[i];
                const bool line = TR ? k[i] < left_k : e[i] < left_rows;
                held[which][i] = u32x4{};
                if (line && there >= kChunk) {
                    using Any = uint32_t __attribute__((ext_vector_type(4), aligned(sizeof(T))));
                    held[which][i] = *(const REX_GLOBAL Any *)(origin + off[i]);
                } else if (line && there > 0) {
                    using Bits = std::conditional_t<kSize == 2, uint16_t, uint32_t>;
                    uint32_t x[kChunk];
#pragma unroll
                    for (int c = 0; c < kChunk; ++c) x[c] = c < there ? as_global<Bits>(origin + off[i])[c] : Bits(0);
#pragma unroll
                    for (int c = 0; c < 4; ++c) {
                        if constexpr (kSize == 2) held[which][i][c] = x[2 * c] | x[2 * c + 1] << 16;
                        else held[which][i][c] = x[c];
                    }
                }
            }
        }
        origin += step_bytes;
        left_k -= kStep;
    }
    __device__ __forceinline__ void put(char *to, int wave, int lane, int which) const {
        if constexpr (!WHOLE) {
#pragma unroll
            for (int i = 0; i < kLoads; ++i)
                *reinterpret_cast<u32x4 *>(to + ((i * WAVES + wave) * 64 + lane) * 16) = held[which][i];
        }
    }

    // Operands of half s of a step, product t of the wave whose first row is `base`.
    struct Reader {
        int at[TR ? 1 : 2], tile, g;
        __device__ __forceinline__ Reader(int base, int lane) {
            const int n = lane & 15;              // row or column of a product
            g = lane >> 4;                        // which chunk of k
            tile = base / 16;
            if constexpr (!TR) {
#pragma unroll
                for (int s = 0; s < 2; ++s) at[s] = (base + n) * 128 + ((4 * s + g) ^ turn(base + n)) * 16;
            } else if constexpr (kSize == 2) {    // sixteen lanes transpose four lines
                at[0] = (8 * g + (n >> 2)) * kPitch + (n >> 1 & 1) * 16 + (n & 1) * 8;
                g = turn(8 * g + (n >> 2)) / 2;
            } else {
                at[0] = 4 * g * kPitch + n * 4;
            }
        }
        __device__ __forceinline__ Frag get(const char *data, int t, int s) const {
            Place p = (Place)(const_cast<char *>(data));
            if constexpr (!TR) {
                return *(const REX_LDS Frag *)(p + at[s] + t * 2048);
            } else if constexpr (kSize == 2) {
#ifdef __HIP_DEVICE_COMPILE__
                using s16x4 = short __attribute__((ext_vector_type(4)));
                using s16x8 = short __attribute__((ext_vector_type(8)));
                s16x4 x[2];
#pragma unroll
                for (int e = 0; e < 2; ++e)
                    x[e] = __builtin_amdgcn_ds_read_tr16_b64_v4i16(
                        (REX_LDS s16x4 *)(p + at[0] + ((tile + t) ^ g) * 32 + (32 * s + 4 * e) * kPitch));
                return __builtin_bit_cast(Frag, s16x8{x[0][0], x[0][1], x[0][2], x[0][3], x[1][0], x[1][1], x[1][2], x[1][3]});
#else
                return Frag{};
#endif
            } else {
                Frag f;
#pragma unroll
                for (int j = 0; j < 4; ++j)
                    f[j] = *(const REX_LDS float *)(p + at[0] + ((tile + t) ^ g) * 64 + (16 * s + j) * kPitch);
                return f;
            }
        }
    };
};

// WM x WN waves of MT x NT products each.
template <typename T, bool TP, bool TQ, int MT, int NT, int WM, int WN, bool WHOLE, int OCC>
__global__ __launch_bounds__(64 * WM * WN, OCC) void gemm_kernel(GemmArgs a) {
    constexpr int kWaves = WM * WN, kRows = 16 * MT, kCols = 16 * NT, BM = kRows * WM, BN = kCols * WN;
    using P = Side<T, TP, BN, kWaves, WHOLE>;
    using Q = Side<T, TQ, BM, kWaves, WHOLE>;
    using Frag = typename P::Frag;
    __shared__ __attribute__((aligned(16))) char smem[2][P::kBytes + Q::kBytes];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    // First the tiles that are made whole, then the parts of the others.  Workgroups go to the eight XCDs
    // in turn: each takes a run of neighbouring tiles, in groups of eight rows of tiles, whose operands
    // its L2 then holds.
    const bool parted = static_cast<int>(blockIdx.x) >= a.grid_whole;
    const int block = blockIdx.x - (parted ? a.grid_whole : 0), some = parted ? a.parted * a.split : a.whole;
    int id = (block & 7) * ((some + 7) >> 3) + (block >> 3);
    if ((block >> 3) >= ((some + 7) >> 3) || id >= some) return;
    const int part = parted ? id / a.parted : 0, rest = parted ? id % a.parted : 0;
    if (parted) id = a.whole + rest;
    const int band = id / (8 * a.tiles_n), rows_of = min(8, a.tiles_m - 8 * band);
    id -= band * 8 * a.tiles_n;
    const int m0 = (8 * band + id % rows_of) * BM, n0 = id / rows_of * BN;

    const int k_steps = (a.K + P::kStep - 1) / P::kStep;
    const int first = parted ? part * a.steps : 0, steps = parted ? min(a.steps, k_steps - first) : k_steps;
    const int k0 = first * P::kStep;
    P p(a.p, a.ldp, n0, a.N, k0, a.K, wave, lane);
    Q q(a.q, a.ldq, m0, a.M, k0, a.K, wave, lane);
    const int wn = wave % WN, wm = wave / WN;
    const typename P::Reader pr(wn * kCols, lane);
    const typename Q::Reader qr(wm * kRows, lane);

    f32x4 acc[MT][NT] = {};
    p.load(smem[0], wave);
    q.load(smem[0] + P::kBytes, wave);
    if (!WHOLE && steps > 1) {
        p.load(nullptr, wave, 1);
        q.load(nullptr, wave, 1);
    }
    // One step, of buffer `which`.  Operands that are not whole chunks come through registers, two steps
    // ahead; the others straight to LDS, one step ahead.
    const auto run = [&](int step, int which) {
        char *now = smem[which], *then = smem[which ^ 1];
        p.put(now, wave, lane, which);
        q.put(now + P::kBytes, wave, lane, which);
        // what this wave loaded is there, and what it read of the other buffer is back
        if (WHOLE) asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
        asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
        __builtin_amdgcn_s_barrier();
        asm volatile("" ::: "memory");
        // (all of a step's reads before the next step's loads: the compiler takes those for writes to
        // what is read, and would wait)
        Frag pf[2][NT], qf[2][MT];
#pragma unroll
        for (int s = 0; s < 2; ++s) {
#pragma unroll
            for (int t = 0; t < NT; ++t) pf[s][t] = pr.get(now, t, s);
#pragma unroll
            for (int t = 0; t < MT; ++t) qf[s][t] = qr.get(now + P::kBytes, t, s);
        }
        if (step + (WHOLE ? 1 : 2) < steps) {
            p.load(then, wave, which);
            q.load(then + P::kBytes, wave, which);
        }
#pragma unroll
        for (int s = 0; s < 2; ++s)
#pragma unroll
            for (int e = 0; e < Shape<T>::kParts; ++e)      // (no product needs the one before it)
#pragma unroll
                for (int i = 0; i < MT; ++i)
#pragma unroll
                    for (int j = 0; j < NT; ++j) acc[i][j] = Shape<T>::mma(pf[s][j], qf[s][i], acc[i][j], e);
    };
    if constexpr (WHOLE) {
        for (int step = 0; step < steps; ++step) run(step, step & 1);
    } else {
        for (int step = 0; step < steps; step += 2) {
            run(step, 0);
            if (step + 1 < steps) run(step + 1, 1);
        }
    }
    // (the compiler leaves out the wait states between products and a use behind a branch)
    asm volatile("s_nop 15" ::: "memory");

    // Results go through LDS, each wave's to a place of its own, so that a row's are written by
    // neighbouring lanes and the epilogue is there once.  16-byte chunks are spread over the banks by
    // their row.
    // A lane's columns are the same in every row that it writes.
    constexpr int kFit = static_cast<int>(sizeof(smem)) / (16 * kCols * 4 * kWaves);
    constexpr int kRound = MT <= kFit ? MT : MT / 2, kQuads = kCols / 4, kStride = 64 / kQuads;
    static_assert(kRound <= kFit && MT % kRound == 0, "results of a round");
    __builtin_amdgcn_s_barrier();
    asm volatile("" ::: "memory");      // (the barrier alone does not hold the stores back)
    f32x4 *stage = reinterpret_cast<f32x4 *>(&smem[0][0]) + wave * kRound * 16 * kQuads;
    const int quad = lane % kQuads, n = n0 + wn * kCols + 4 * quad, left = a.N - n;
    const int wave_m = wm * kRows + lane / kQuads;
    const f32x4 bias = parted ? f32x4{} : load_bias(a, min(n, a.N - 1));
    f32x4 *sums = reinterpret_cast<f32x4 *>(a.part) + (static_cast<int64_t>(part) * a.parted + rest) * (BM * BN / 4) +
                  (wn * kCols >> 2) + quad;
#pragma unroll
    for (int r = 0; r < MT; r += kRound) {
#pragma unroll
        for (int i = 0; i < kRound; ++i) {
            const int row = 16 * i + (lane & 15);
#pragma unroll
            for (int j = 0; j < NT; ++j)
                stage[row * kQuads + ((4 * j + (lane >> 4)) ^ (row & (kQuads - 1)))] = acc[r + i][j];
        }
        asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
        const int m = m0 + wave_m + 16 * r, rows = left > 0 ? a.M - m : 0;
        int64_t at = static_cast<int64_t>(m) * a.N + n, rat = m * a.ldr + n;
#pragma unroll 4
        for (int i = 0; i < 16 * kRound; i += kStride) {
            const int row = i + lane / kQuads;
            const f32x4 x = stage[row * kQuads + (quad ^ (row & (kQuads - 1)))] + bias;
            if (parted) as_global_mut<f32x4>(sums)[(wave_m + 16 * r + i) * (BN / 4)] = x;
            else if (i < rows) finish4<T>(a, left, at, rat, x);
            at += static_cast<int64_t>(kStride) * a.N;
            rat += kStride * a.ldr;
        }
        asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
    }
}

template <typename T, bool TP, bool TQ, int MT, int NT, int WM, int WN, bool WHOLE, int OCC>
hipError_t run_gemm(const GemmArgs &a, hipStream_t s) {
    const uint32_t grid = a.grid_whole + (a.parted * a.split + 7) / 8 * 8;
    gemm_kernel<T, TP, TQ, MT, NT, WM, WN, WHOLE, OCC><<<grid, 64 * WM * WN, 0, s>>>(a);
    return hipGetLastError();
}

}  // namespace rex
