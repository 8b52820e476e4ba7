// epilogue.hpp -- what follows a dense layer's sums: bias, activation and its slope, residual, stores.
#pragma once

#include "attn.hpp"
#include "linear.hpp"

namespace rex {

// ---------------------------------------------------------------------------
// Activations
// ---------------------------------------------------------------------------

// erfc(z) = t R(t) exp(-z^2) for z >= 0, t = 1 / (1 + 0.45 z), R the polynomial of degree nine with
// the least largest relative error over all z (3.2e-8; 3.7e-7 as evaluated here), found by
// reweighted least squares at Chebyshev points.  A relative error, so that the left tail of the
// normal distribution is as exact as the rest.
__device__ __forceinline__ float erfc_over_exp(float z) {
    const float t = __builtin_amdgcn_rcpf(fmaf(0.45f, z, 1.0f));
    float r = -0.041390951722860336f;
    r = fmaf(r, t, 0.19068720936775208f);
    r = fmaf(r, t, -0.30058127641677856f);
    r = fmaf(r, t, 0.14239980280399323f);
    r = fmaf(r, t, -0.022357303649187088f);
    r = fmaf(r, t, 0.11995022743940353f);
    r = fmaf(r, t, 0.17525216937065125f);
    r = fmaf(r, t, 0.22827163338661194f);
    r = fmaf(r, t, 0.25388315320014954f);
    return t * fmaf(r, t, 0.25388532876968384f);
}

// act(x), and its slope at x, of four.
__device__ __forceinline__ void activate(int act, f32x4 &x, float (&slope)[4]) {
    if (act == kActRelu) {                      // NaN stays, and lets the gradient through
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            slope[i] = x[i] <= 0.0f ? 0.0f : 1.0f;
            x[i] = x[i] <= 0.0f ? 0.0f : x[i];
        }
    } else if (act == kActGelu) {               // x Phi(x), Phi + x phi(x)
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const float e = __builtin_amdgcn_exp2f(x[i] * x[i] * (-0.5f * kLog2e));
            const float tail = 0.5f * e * erfc_over_exp(fabsf(x[i]) * 0.70710678118654752f);
            const float phi = x[i] < 0.0f ? tail : 1.0f - tail;
            slope[i] = fmaf(x[i] * 0.39894228040143268f, e, phi);
            x[i] *= phi;
        }
    } else if (act == kActSilu) {               // x s, s (1 + x (1 - s))
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const float s = __builtin_amdgcn_rcpf(1.0f + __builtin_amdgcn_exp2f(-kLog2e * x[i]));
            slope[i] = s * fmaf(x[i], 1.0f - s, 1.0f);
            x[i] *= s;
        }
    }
}

// The slope kept for the backward: binary32 beside binary32 data, and beside bf16 data 24 bits in
// steps of 2^-23 from -1/4 on (slopes lie in [-0.13, 1.13]; 0 and 1 are exact), all ones for NaN: the
// upper 16 of all slopes, then the lower 8 of all.  (16 bits would do for the products, whose operands
// are bf16, but the bias gradient, a binary32 sum over all rows, would be 1.3e-5 of itself off; binary32
// would be a quarter more bytes than 24 bits, and there is nothing to evaluate in the backward.  The step is
// absolute: below x = -5.92 the slope of gelu, and below x = -19.6 that of silu, is under half of it and counts
// as 0.)
template <typename T> struct Slope;
template <> struct Slope<float> {
    template <int V> static __device__ __forceinline__ void store(void *p, int64_t, int64_t at, const float *x) {
        using W = float __attribute__((ext_vector_type(V), aligned(4)));
        W w;
#pragma unroll
        for (int i = 0; i < V; ++i) w[i] = x[i];
        *(REX_GLOBAL W *)(static_cast<float *>(p) + at) = w;
    }
    template <int V> static __device__ __forceinline__ void load(const void *p, int64_t, int64_t at, float *x) {
        using W = float __attribute__((ext_vector_type(V), aligned(4)));
        const W w = *(const REX_GLOBAL W *)(static_cast<const float *>(p) + at);
#pragma unroll
        for (int i = 0; i < V; ++i) x[i] = w[i];
    }
};
template <> struct Slope<uint16_t> {
    // slopes `at` .. at + V - 1 of `all`; V > 1: at and all are multiples of V
    template <int V> static __device__ __forceinline__ void store(void *p, int64_t all, int64_t at, const float *x) {
        using H = uint16_t __attribute__((ext_vector_type(V)));
        using L = uint8_t __attribute__((ext_vector_type(V)));
        H h;
        L l;
#pragma unroll
        for (int i = 0; i < V; ++i) {
            const uint32_t c = static_cast<uint32_t>(fmaf(x[i], 0x1p23f, 0x1p21f + 0.5f));
            const uint32_t u = x[i] != x[i] ? 0xffffffu : c;
            h[i] = static_cast<uint16_t>(u >> 8);
            l[i] = static_cast<uint8_t>(u);
        }
        *(REX_GLOBAL H *)(static_cast<uint16_t *>(p) + at) = h;
        *(REX_GLOBAL L *)(static_cast<uint8_t *>(p) + 2 * all + at) = l;
    }
    template <int V> static __device__ __forceinline__ void load(const void *p, int64_t all, int64_t at, float *x) {
        using H = uint16_t __attribute__((ext_vector_type(V)));
        using L = uint8_t __attribute__((ext_vector_type(V)));
        const H h = *(const REX_GLOBAL H *)(static_cast<const uint16_t *>(p) + at);
        const L l = *(const REX_GLOBAL L *)(static_cast<const uint8_t *>(p) + 2 * all + at);
#pragma unroll
        for (int i = 0; i < V; ++i) {
            const uint32_t u = static_cast<uint32_t>(h[i]) << 8 | l[i];
            x[i] = u == 0xffffffu ? __builtin_nanf("") : fmaf(static_cast<float>(u), 0x1p-23f, -0.25f);
        }
    }
};

template <typename T> __device__ __forceinline__ void load4(const void *p, int64_t at, float (&x)[4]);
template <> __device__ __forceinline__ void load4<float>(const void *p, int64_t at, float (&x)[4]) {
    const f32x4 v = *(const REX_GLOBAL f32x4 *)(static_cast<const float *>(p) + at);
    for (int i = 0; i < 4; ++i) x[i] = v[i];
}
template <> __device__ __forceinline__ void load4<uint16_t>(const void *p, int64_t at, float (&x)[4]) {
    const u32x2 v = *(const REX_GLOBAL u32x2 *)(static_cast<const uint16_t *>(p) + at);
    for (int i = 0; i < 4; ++i) x[i] = __uint_as_float(i & 1 ? v[i >> 1] & 0xffff0000u : v[i >> 1] << 16);
}

// The biases of columns n .. n + 3 (0 where there is none).
__device__ __forceinline__ f32x4 load_bias(const GemmArgs &a, int n) {
    f32x4 x = {};
    if (!a.bias) return x;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const int at = min(n + i, a.N - 1);
        x[i] = a.bias_bf16 ? bf16_to_f32(as_global<uint16_t>(a.bias)[at]) : as_global<float>(a.bias)[at];
    }
    return x;
}

// Four adjacent results (`left` of them, if there are fewer) at element `at` of the dense results,
// whose sums are x: activation, residual (at element `rat`), stores.
template <typename T>
__device__ __forceinline__ void finish4(const GemmArgs &a, int left, int64_t at, int64_t rat, f32x4 x) {
    float s[4], r[4] = {};
    if (a.vec) {                        // (then N is a multiple of 4)
        if (a.residual) load4<T>(a.residual, rat, r);
        if (a.act != kActNone) activate(a.act, x, s);
        if (a.residual) {
#pragma unroll
            for (int i = 0; i < 4; ++i) x[i] += r[i];
        }
        Num<T>::store4(reinterpret_cast<char *>(static_cast<T *>(a.out) + at), x);
        if (a.slope) Slope<T>::template store<4>(a.slope, static_cast<int64_t>(a.M) * a.N, at, s);
        return;
    }
    if (a.act != kActNone) activate(a.act, x, s);
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        if (i >= left) break;
        if (a.residual) x[i] += load_f32<T>(as_global<T>(a.residual) + rat + i);
        store_f32<T>(as_global_mut<T>(a.out) + at + i, x[i]);
        if (a.slope) Slope<T>::template store<1>(a.slope, static_cast<int64_t>(a.M) * a.N, at + i, s + i);
    }
}

}  // namespace rex
