// memory.hip -- the 8-bit memory of boxes: quantising as it is written, reading back
// (box_memory_append, box_memory_read; the attention over it is attn_fwd.hpp).
//
// Sixteen lanes take one (box, key head), eight channels each; both are bound by the bytes
// they move.
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

dim3 memory_grid(const MemoryArgs &a) {
    return dim3(static_cast<uint32_t>((a.count * a.Hkv * kLanes + 255) / 256));
}

}  // namespace

hipError_t launch_memory_append(const MemoryArgs &a, int dtype, hipStream_t s) {
    if (dtype == kBF16) hipLaunchKernelGGL((memory_append_kernel<uint16_t>), memory_grid(a), dim3(256), 0, s, a);
    else hipLaunchKernelGGL((memory_append_kernel<float>), memory_grid(a), dim3(256), 0, s, a);
    return hipGetLastError();
}

hipError_t launch_memory_read(const MemoryArgs &a, int dtype, hipStream_t s) {
    if (dtype == kBF16) hipLaunchKernelGGL((memory_read_kernel<uint16_t>), memory_grid(a), dim3(256), 0, s, a);
    else hipLaunchKernelGGL((memory_read_kernel<float>), memory_grid(a), dim3(256), 0, s, a);
    return hipGetLastError();
}

}  // namespace rex
