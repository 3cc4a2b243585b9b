// glu_device.hpp -- what the gated feed-forward kernels share: the activations
// with their derivatives, and the matrix cores' operands of each storage type.
#pragma once

#include "device.hpp"
#include "internal.h"
#include "mx_device.hpp"

namespace exemcl {

// ---------------------------------------------------------------------------
// Activations.  sigma(z) = 1 / (1 + e^-z); FAST (results of 16 bits): the
// exponential and the reciprocal of the instructions, together within 2^-19 of
// the value for |z| < 64 (the argument's own rounding, z log2 e 2^-24, is most of
// it), against the 2^-12 at least of the result's type.
// ---------------------------------------------------------------------------
template <bool FAST>
__device__ __forceinline__ float sigma(float z) {
    if constexpr (FAST) return __builtin_amdgcn_rcpf(1.0f + __builtin_amdgcn_exp2f(z * -1.44269504088896341f));
    return 1.0f / (1.0f + expf(-z));
}

// a(g) and, where SLOPE, its derivative.
//   silu       a = g s, a' = s + g s (1 - s), s = sigma(g)
//   gelu       a = g P, a' = P + g e^(-g^2 / 2) / sqrt(2 pi), P = erfc(-g / sqrt 2) / 2
//   gelu_tanh  a = g s, a' = s + g s (1 - s) 2 z', s = sigma(2 z) = (1 + tanh z) / 2,
//              z = sqrt(2 / pi) (g + 0.044715 g^3)
//   relu       a = max(g, 0), a' = 1 where g > 0
// A factor that is 0 makes its term 0, also where g is infinite.
template <int ACT, bool FAST, bool SLOPE>
__device__ __forceinline__ float activation(float g, float &slope) {
    if constexpr (ACT == ACT_RELU) {
        if constexpr (SLOPE) slope = g > 0.0f ? 1.0f : g == g ? 0.0f : g;
        return g > 0.0f ? g : g == g ? 0.0f : g;
    } else {
        float s, t;  // the factor of g, and that of g in the derivative
        if constexpr (ACT == ACT_SILU) {
            s = sigma<FAST>(g);
            t = s * (1.0f - s);
        } else if constexpr (ACT == ACT_GELU_TANH) {
            const float g2 = g * g;
            s = sigma<FAST>(1.59576912160573071f * g * fmaf(0.044715f, g2, 1.0f));
            t = s * (1.0f - s);
            if constexpr (SLOPE) t = t > 0.0f ? t * 1.59576912160573071f * fmaf(0.134145f, g2, 1.0f) : 0.0f;
        } else {
            s = 0.5f * erfcf(-0.707106781186547524f * g);
            t = 0.0f;
            if constexpr (SLOPE) t = 0.398942280401432678f * (FAST ? __builtin_amdgcn_exp2f(g * g * -0.72134752044448170f) : expf(-0.5f * g * g));
        }
        if constexpr (SLOPE) slope = t != 0.0f ? fmaf(g, t, s) : s;
        return s != 0.0f ? g * s : 0.0f;
    }
}

template <int ACT, bool FAST>
__device__ __forceinline__ float activation(float g) {
    float unused;
    return activation<ACT, FAST, false>(g, unused);
}

// Calls f with the activation as a constant.
template <typename F>
__device__ __forceinline__ void with_activation(int act, F &&f) {
    if (act == ACT_SILU)
        f(std::integral_constant<int, ACT_SILU>());
    else if (act == ACT_GELU)
        f(std::integral_constant<int, ACT_GELU>());
    else if (act == ACT_GELU_TANH)
        f(std::integral_constant<int, ACT_GELU_TANH>());
    else
        f(std::integral_constant<int, ACT_RELU>());
}

// ---------------------------------------------------------------------------
// Operands.  16-bit values are the instructions' own; an fp32 value is the sum of
// three bf16 ones (hi + mid + lo, each the rounding of what is left), and a
// product of two the six products of parts that are not below 2^-27 of it, added
// in the fp32 accumulators: 2.7 times the fp32 instruction's rate.  A value that
// rounds to an infinity keeps its upper bits instead, and an infinity or NaN
// has no other parts.
// ---------------------------------------------------------------------------
__device__ __forceinline__ void split_parts(float x, __bf16 &hi, __bf16 &mid, __bf16 &lo) {
    const uint32_t bits = __float_as_uint(x);
    __bf16 h = (__bf16)x;
    if ((bits & 0x7fffffffu) >= 0x7f7f8000u)  // past the largest bf16
        h = __builtin_bit_cast(__bf16, (uint16_t)((bits >> 16) | ((bits & 0x7fffffffu) > 0x7f800000u ? 0x40u : 0u)));
    const float r = (bits & 0x7f800000u) == 0x7f800000u ? 0.0f : x - (float)h;
    hi = h;
    mid = (__bf16)r;
    lo = (__bf16)(r - (float)mid);
}

template <typename T>
struct Operand {  // fp16, bf16
    using E = T;
    static constexpr int PARTS = 1, PRODUCTS = 1;
};
template <>
struct Operand<float> {
    using E = __bf16;
    static constexpr int PARTS = 3, PRODUCTS = 6;
};
// Parts of product p of an fp32 product, each in two bits: (hi, hi), (hi, mid),
// (mid, hi), (hi, lo), (lo, hi), (mid, mid).
constexpr uint32_t kPartsA = 0u | 0u << 2 | 1u << 4 | 0u << 6 | 2u << 8 | 1u << 10;
constexpr uint32_t kPartsB = 0u | 1u << 2 | 0u << 4 | 2u << 6 | 0u << 8 | 1u << 10;
__host__ __device__ constexpr int part_a(int p) { return kPartsA >> (2 * p) & 3; }
__host__ __device__ constexpr int part_b(int p) { return kPartsB >> (2 * p) & 3; }

// Four results in a row, `have` of them inside it.
template <typename T>
__device__ __forceinline__ void store4(T *p, int have, const float (&v)[4]) {
    typedef T vec __attribute__((ext_vector_type(4), aligned(sizeof(T))));
    if (have >= 4) {
        vec x;
#pragma unroll
        for (int i = 0; i < 4; ++i) x[i] = (T)v[i];
        *reinterpret_cast<vec *>(p) = x;
    } else {
#pragma unroll
        for (int i = 0; i < 3; ++i)
            if (i < have) p[i] = (T)v[i];
    }
}

}  // namespace exemcl
