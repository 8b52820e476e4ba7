// memory.hip -- the 8-bit memory of boxes: quantising as it is written, reading back
// (box_memory_append, box_memory_read; the attention over it is attn_fwd.hpp).
//
// Sixteen lanes take one (box, key head), eight channels each.  Keys lie in the memory as rows
// of channels, values as rows of places (what the attention's product reads), so a box's values
// are one byte in each of dim rows, and it is the number of those accesses that bounds a call,
// not its bytes.  There are two forms:
//   few boxes    one launch over (box, head), each byte an access of its own;
//   many boxes   a workgroup owns some pages, finds the call's boxes in them by reading all slots
//                (8 bytes a box, from L2), and each of its waves takes a (page, head): the values
//                pass through LDS, and 64 adjacent bytes of the page are one access.
// Shuffled slots, 2048 pages, 16 heads of 64 channels, 16000 boxes, append / read, us: binary32 134 / 102
// the first way and 89 / 53 the second (the same slots read back; others: 101 / 66), bf16 123 / 92 and
// 93 / 42; 4000 boxes 38 / 28 and 48 / 26.  bf16, 32768 pages, 16000 boxes in 8 heads of 64: 74 / 50 and
// 177 / 110; 512 pages, 16000 boxes in 8 heads of 32: 34 / 18 and 38 / 18.  So the second takes a call
// with four boxes for each page of the memory and 2^23 values, where there are pages enough for its
// workgroups.  Its 16000 boxes are 333 MB both ways, 68 us at the rate of a large copy.  What bounds it is
// latency: a wave's (page, head) has few boxes, and each goes from its slot over its row to LDS and
// to the page (with slots in order 61 / 38).
#include <algorithm>

#include "attn.hpp"

namespace rex {

namespace {

constexpr int kLanes = 16;    // 8 channels each: 128

// Eight channels of a row of any alignment.
template <typename T>
__device__ __forceinline__ void load8(const void *p, int64_t at, bool vec, float (&x)[8]) {
    if (vec) {
        const auto f = Num<T>::load(static_cast<const char *>(p) + at * Num<T>::kSize);
#pragma unroll
        for (int i = 0; i < 8; ++i) x[i] = static_cast<float>(f[i]);
    } else {
#pragma unroll
        for (int i = 0; i < 8; ++i) x[i] = load_f32<T>(as_global<T>(p) + at + i);
    }
}

// Codes of eight channels and the scale of all 128 (every lane of the sixteen has it).
// One rounding per written operation: the codes are defined by these binary32 steps.
__device__ __forceinline__ float encode(const float (&x)[8], int (&code)[8]) {
    float top = 0.0f;
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        const float v = fabsf(x[i]);
        top = v < kInf ? fmaxf(top, v) : top;     // false for NaN too
    }
#pragma unroll
    for (int d = 1; d < kLanes; d <<= 1) top = fmaxf(top, __shfl_xor(top, d));
    const float scale = top / 127.0f;
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        const float q = fminf(fmaxf(rintf(x[i] / scale), -127.0f), 127.0f);
        code[i] = scale == 0.0f || x[i] != x[i] ? 0 : static_cast<int>(q);
    }
    return scale;
}

template <typename T>
__global__ __launch_bounds__(256) void memory_append_kernel(MemoryArgs a) {
    const int64_t e = (static_cast<int64_t>(blockIdx.x) * 256 + threadIdx.x) / kLanes;
    const int c = threadIdx.x & (kLanes - 1), ch = 8 * c;
    if (e >= a.count * a.Hkv) return;             // whole groups of sixteen lanes
    const int64_t i = e / a.Hkv;
    const int h = static_cast<int>(e - i * a.Hkv);
    const int64_t slot = as_global<int64_t>(a.slots)[i];
    if (slot < 0 || slot >= a.num_slots) return;
    const int64_t page = slot / kTile;
    const int at = static_cast<int>(slot - page * kTile);
    const int64_t ph = page * a.Hkv + h;
    float x[8] = {};
    int code[8];
    if (ch < a.D) load8<T>(a.k, i * a.k_sr + h * a.k_sh + ch, a.vec, x);
    float scale = encode(x, code);
    if (ch < a.D) {
        u32x2 w = {};
#pragma unroll
        for (int j = 0; j < 8; ++j) w[j >> 2] |= (static_cast<uint32_t>(code[j]) & 0xffu) << (8 * (j & 3));
        *(REX_GLOBAL u32x2 *)(a.k8 + (ph * kTile + at) * a.D + ch) = w;
    }
    if (c == 0) as_global_mut<float>(a.ks)[ph * kTile + at] = scale;
    if (ch < a.D) load8<T>(a.v, i * a.v_sr + h * a.v_sh + ch, a.vec, x);
    scale = encode(x, code);
    if (ch < a.D) {
#pragma unroll
        for (int j = 0; j < 8; ++j)
            as_global_mut<int8_t>(a.v8)[(ph * a.D + ch + j) * kTile + at] = static_cast<int8_t>(code[j]);
    }
    if (c == 0) as_global_mut<float>(a.vs)[ph * kTile + at] = scale;
    if (h == 0 && c < 4)
        as_global_mut<float>(a.mbox)[slot * 4 + c] = as_global<float>(a.boxes)[i * 4 + c];
}

template <typename T>
__global__ __launch_bounds__(256) void memory_read_kernel(MemoryArgs a) {
    using N = Num<T>;
    const int64_t e = (static_cast<int64_t>(blockIdx.x) * 256 + threadIdx.x) / kLanes;
    const int c = threadIdx.x & (kLanes - 1), ch = 8 * c;
    if (e >= a.count * a.Hkv) return;
    const int64_t i = e / a.Hkv;
    const int h = static_cast<int>(e - i * a.Hkv);
    const int64_t slot = as_global<int64_t>(a.slots)[i];
    const bool there = slot >= 0 && slot < a.num_slots;
    const int64_t page = there ? slot / kTile : 0;
    const int at = there ? static_cast<int>(slot - page * kTile) : 0;
    const int64_t ph = page * a.Hkv + h;
    float x[8] = {};
    if (ch < a.D && a.k_out) {
        if (there) {
            const float s = as_global<float>(a.ks)[ph * kTile + at];
            const u32x2 w = *(const REX_GLOBAL u32x2 *)(a.k8 + (ph * kTile + at) * a.D + ch);
#pragma unroll
            for (int j = 0; j < 8; ++j)
                x[j] = static_cast<float>(static_cast<int8_t>(w[j >> 2] >> (8 * (j & 3)))) * s;
        }
        N::store(static_cast<char *>(a.k_out) + (e * a.D + ch) * N::kSize, x);
    }
    if (ch < a.D && a.v_out) {
        if (there) {
            const float s = as_global<float>(a.vs)[ph * kTile + at];
#pragma unroll
            for (int j = 0; j < 8; ++j)
                x[j] = static_cast<float>(as_global<int8_t>(a.v8)[(ph * a.D + ch + j) * kTile + at]) * s;
        }
        N::store(static_cast<char *>(a.v_out) + (e * a.D + ch) * N::kSize, x);
    }
    if (a.boxes_out && h == 0 && c < 4)
        as_global_mut<float>(a.boxes_out)[i * 4 + c] =
            there ? as_global<float>(a.mbox)[slot * 4 + c] : 0.0f;
}

// ---------------------------------------------------------------------------
// Many boxes: workgroup w owns pages w, w + kOwners, ...
// ---------------------------------------------------------------------------

constexpr int kOwners = 512, kOwned = 256;      // workgroups, and the most pages of one
// Fewer pages leave most workgroups without one: 16000 reads in binary32, 8 heads of 128 channels, of
// 128 pages 48 us (each box by itself 53), of 64 pages 74 (47), of 16 208 (47), of one 3206 (46).
constexpr int kFewPages = 128;
constexpr int64_t kManyValues = 1 << 23;
constexpr int kOwnWaves = 16, kOwnThreads = kOwnWaves * 64;
constexpr int kRow = kTile + 4;                 // bytes of a row of a page's values in LDS
constexpr int kSlotLoads = 2;                   // slots that a thread has on their way
constexpr int kList = 2 * kSlotLoads * kOwnThreads;

// The places of the set bits of `m`, in order.
__device__ __forceinline__ int ranked(uint64_t m, int lane, uint8_t *order) {
    if (m >> lane & 1) order[__popcll(m & ((uint64_t(1) << lane) - 1))] = static_cast<uint8_t>(lane);
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
    return __popcll(m);
}

template <typename T>
__global__ __launch_bounds__(kOwnThreads) void memory_append_pages_kernel(MemoryArgs a) {
    extern __shared__ char smem[];
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    const int owned = a.owned, count = static_cast<int>(a.count);
    int *const item = reinterpret_cast<int *>(smem);           // the call's box for each owned place
    uint8_t *const order = reinterpret_cast<uint8_t *>(item + owned * kTile) + wave * 64;
    char *const tile = smem + owned * kTile * 4 + kOwnWaves * 64 + wave * a.D * kRow;
    for (int i = tid; i < owned * kTile; i += kOwnThreads) item[i] = -1;
    __syncthreads();
    for (int base = 0; base < count; base += 4 * kOwnThreads) {
        int64_t slot[4];
#pragma unroll
        for (int u = 0; u < 4; ++u) {
            const int i = base + u * kOwnThreads + tid;
            slot[u] = i < count ? as_global<int64_t>(a.slots)[i] : -1;
        }
#pragma unroll
        for (int u = 0; u < 4; ++u) {
            const int64_t page = slot[u] / kTile;
            if (slot[u] >= 0 && slot[u] < a.num_slots && page % kOwners == blockIdx.x)
                atomicMax(item + page / kOwners * kTile + slot[u] % kTile, base + u * kOwnThreads + tid);
        }
    }
    __syncthreads();
    for (int e = tid; e < owned * kTile * 4; e += kOwnThreads) {
        const int i = item[e / 4];
        if (i < 0) continue;
        const int64_t page = static_cast<int64_t>(e / (4 * kTile)) * kOwners + blockIdx.x;
        as_global_mut<float>(a.mbox)[page * kTile * 4 + e % (4 * kTile)] = as_global<float>(a.boxes)[static_cast<int64_t>(i) * 4 + e % 4];
    }
    const int c = lane & (kLanes - 1), ch = 8 * c;
    for (int unit = wave; unit < owned * a.Hkv; unit += kOwnWaves) {
        const int p = unit / a.Hkv, h = unit - p * a.Hkv;
        const uint32_t mask = static_cast<uint32_t>(__ballot(lane < kTile && item[p * kTile + lane % kTile] >= 0));
        if (mask == 0) continue;
        const int n = ranked(mask, lane, order);
        const int64_t ph = (static_cast<int64_t>(p) * kOwners + blockIdx.x) * a.Hkv + h;
        for (int j0 = 0; j0 < n; j0 += 4) {
            const int j = j0 + lane / kLanes;
            const bool on = j < n && ch < a.D;
            const int at = order[min(j, n - 1)];
            const int64_t i = item[p * kTile + at];
            float x[2][8] = {};
            if (on) {
                load8<T>(a.k, i * a.k_sr + h * a.k_sh + ch, a.vec, x[0]);
                load8<T>(a.v, i * a.v_sr + h * a.v_sh + ch, a.vec, x[1]);
            }
            int code[8];
            float scale = encode(x[0], code);
            if (on) {
                u32x2 w = {};
#pragma unroll
                for (int e = 0; e < 8; ++e) w[e >> 2] |= (static_cast<uint32_t>(code[e]) & 0xffu) << (8 * (e & 3));
                *(REX_GLOBAL u32x2 *)(a.k8 + (ph * kTile + at) * a.D + ch) = w;
                if (c == 0) as_global_mut<float>(a.ks)[ph * kTile + at] = scale;
            }
            scale = encode(x[1], code);
            if (on) {
#pragma unroll
                for (int e = 0; e < 8; ++e) tile[(ch + e) * kRow + at] = static_cast<char>(code[e]);
                if (c == 0) as_global_mut<float>(a.vs)[ph * kTile + at] = scale;
            }
        }
        __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
        int8_t *const v8 = a.v8 + ph * a.D * kTile;
        if (mask == 0xffffffffu) {
            for (int r = lane >> 1; r < a.D; r += 32) {
                const uint32_t *src = reinterpret_cast<const uint32_t *>(tile + r * kRow + (lane & 1) * 16);
                *(REX_GLOBAL u32x4 *)(v8 + r * kTile + (lane & 1) * 16) = u32x4{src[0], src[1], src[2], src[3]};
            }
        } else if (mask >> (lane % kTile) & 1) {
            // (bytes: the other places of the page may be written by another call meanwhile)
            for (int r = lane / kTile; r < a.D; r += 2)
                as_global_mut<int8_t>(v8)[r * kTile + lane % kTile] = tile[r * kRow + lane % kTile];
        }
        __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
    }
}

template <typename T>
__global__ __launch_bounds__(kOwnThreads) void memory_read_pages_kernel(MemoryArgs a) {
    using N = Num<T>;
    extern __shared__ char smem[];
    __shared__ int listed;
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    const int owned = a.owned, count = static_cast<int>(a.count);
    // the boxes found, (number in the call, owned page * 32 + place), and how many of each page;
    // page `owned` stands for the slots outside the memory
    int *const num = reinterpret_cast<int *>(smem);
    int *const found = num + kList, *const place = found + kList;
    uint8_t *const order = reinterpret_cast<uint8_t *>(place + (owned + 4) / 4 * 4) + wave * 64;
    char *const tile = reinterpret_cast<char *>(place + (owned + 4) / 4 * 4) + kOwnWaves * 64 + wave * a.D * kRow;
    const int c = lane & (kLanes - 1), ch = 8 * c;

    auto read = [&](int n) {
        if (a.boxes_out)
            for (int e = tid; e < n * 4; e += kOwnThreads) {
                const int key = found[e / 4], p = key / kTile;
                const int64_t slot = (static_cast<int64_t>(p) * kOwners + blockIdx.x) * kTile + key % kTile;
                as_global_mut<float>(a.boxes_out)[static_cast<int64_t>(num[e / 4]) * 4 + e % 4] =
                    p < owned ? as_global<float>(a.mbox)[slot * 4 + e % 4] : 0.0f;
            }
        for (int unit = wave; unit < (owned + 1) * a.Hkv; unit += kOwnWaves) {
            const int p = unit / a.Hkv, h = unit - p * a.Hkv;
            if (place[p] == 0) continue;
            const bool there = p < owned;
            const int64_t ph = (static_cast<int64_t>(p) * kOwners + blockIdx.x) * a.Hkv + h;
            if (there && a.v_out) {
                for (int r = lane >> 1; r < a.D; r += 32) {
                    const u32x4 x = *(const REX_GLOBAL u32x4 *)(a.v8 + (ph * a.D + r) * kTile + (lane & 1) * 16);
                    uint32_t *dst = reinterpret_cast<uint32_t *>(tile + r * kRow + (lane & 1) * 16);
#pragma unroll
                    for (int e = 0; e < 4; ++e) dst[e] = x[e];
                }
            }
            __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
            for (int l0 = 0; l0 < n; l0 += 64) {
                const int m = ranked(__ballot(l0 + lane < n && found[min(l0 + lane, n - 1)] / kTile == p), lane, order);
                for (int j0 = 0; j0 < m; j0 += 4) {
                    const int j = j0 + lane / kLanes;
                    if (j >= m || ch >= a.D) continue;
                    const int l = l0 + order[j], at = found[l] % kTile;
                    const int64_t to = ((static_cast<int64_t>(num[l]) * a.Hkv + h) * a.D + ch) * N::kSize;
                    float x[8] = {};
                    if (a.k_out) {
                        if (there) {
                            const float s = as_global<float>(a.ks)[ph * kTile + at];
                            const u32x2 w = *(const REX_GLOBAL u32x2 *)(a.k8 + (ph * kTile + at) * a.D + ch);
#pragma unroll
                            for (int e = 0; e < 8; ++e)
                                x[e] = static_cast<float>(static_cast<int8_t>(w[e >> 2] >> (8 * (e & 3)))) * s;
                        }
                        N::store(static_cast<char *>(a.k_out) + to, x);
                    }
                    if (a.v_out) {
                        if (there) {
                            const float s = as_global<float>(a.vs)[ph * kTile + at];
#pragma unroll
                            for (int e = 0; e < 8; ++e)
                                x[e] = static_cast<float>(static_cast<int8_t>(tile[(ch + e) * kRow + at])) * s;
                        }
                        N::store(static_cast<char *>(a.v_out) + to, x);
                    }
                }
                __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
            }
        }
    };

    auto empty = [&]() {
        if (tid == 0) listed = 0;
        for (int i = tid; i <= owned; i += kOwnThreads) place[i] = 0;
        __syncthreads();
    };
    empty();
    for (int base = 0; base < count; base += kSlotLoads * kOwnThreads) {
        int64_t slot[kSlotLoads];
#pragma unroll
        for (int u = 0; u < kSlotLoads; ++u) {
            const int i = base + u * kOwnThreads + tid;
            slot[u] = i < count ? as_global<int64_t>(a.slots)[i] : 0;
        }
        __syncthreads();
        const int n = listed;             // kSlotLoads * kOwnThreads more have room in half the list
        __syncthreads();
        if (n > kList / 2) {
            read(n);
            __syncthreads();
            empty();
        }
#pragma unroll
        for (int u = 0; u < kSlotLoads; ++u) {
            const int i = base + u * kOwnThreads + tid;
            if (i >= count) continue;
            const bool there = slot[u] >= 0 && slot[u] < a.num_slots;
            const int64_t page = there ? slot[u] / kTile : i;
            if (page % kOwners != blockIdx.x) continue;
            const int p = there ? static_cast<int>(page / kOwners) : owned;
            const int l = atomicAdd(&listed, 1);
            num[l] = i;
            found[l] = p * kTile + (there ? static_cast<int>(slot[u] % kTile) : 0);
            atomicAdd(place + p, 1);
        }
    }
    __syncthreads();
    read(listed);
}

dim3 memory_grid(const MemoryArgs &a) {
    return dim3(static_cast<uint32_t>((a.count * a.Hkv * kLanes + 255) / 256));
}

// Whether the pages' owners do the work, and how many pages each has then.
bool by_pages(MemoryArgs &a) {
    const int64_t owned = (a.num_slots / kTile + kOwners - 1) / kOwners;
    a.owned = static_cast<int32_t>(std::min<int64_t>(owned, kOwned));
    return a.num_slots >= kFewPages * kTile && owned <= kOwned && a.count * kTile >= 4 * a.num_slots && a.count * a.Hkv * a.D >= kManyValues;
}

}  // namespace

hipError_t launch_memory_append(MemoryArgs a, int dtype, hipStream_t s) {
    if (by_pages(a)) {
        const size_t lds = a.owned * kTile * 4 + kOwnWaves * (64 + a.D * kRow);
        if (dtype == kBF16) hipLaunchKernelGGL((memory_append_pages_kernel<uint16_t>), dim3(kOwners), dim3(kOwnThreads), lds, s, a);
        else hipLaunchKernelGGL((memory_append_pages_kernel<float>), dim3(kOwners), dim3(kOwnThreads), lds, s, a);
    } else {
        if (dtype == kBF16) hipLaunchKernelGGL((memory_append_kernel<uint16_t>), memory_grid(a), dim3(256), 0, s, a);
        else hipLaunchKernelGGL((memory_append_kernel<float>), memory_grid(a), dim3(256), 0, s, a);
    }
    return hipGetLastError();
}

hipError_t launch_memory_read(MemoryArgs a, int dtype, hipStream_t s) {
    if (by_pages(a)) {
        const size_t lds = (2 * kList + (a.owned + 4) / 4 * 4) * 4 + kOwnWaves * (64 + a.D * kRow);
        if (dtype == kBF16) hipLaunchKernelGGL((memory_read_pages_kernel<uint16_t>), dim3(kOwners), dim3(kOwnThreads), lds, s, a);
        else hipLaunchKernelGGL((memory_read_pages_kernel<float>), dim3(kOwners), dim3(kOwnThreads), lds, s, a);
    } else {
        if (dtype == kBF16) hipLaunchKernelGGL((memory_read_kernel<uint16_t>), memory_grid(a), dim3(256), 0, s, a);
        else hipLaunchKernelGGL((memory_read_kernel<float>), memory_grid(a), dim3(256), 0, s, a);
    }
    return hipGetLastError();
}

}  // namespace rex
