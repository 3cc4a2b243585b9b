// glu_device.hpp -- what the gated feed-forward kernels share: the activations
// with their derivatives, and the matrix cores' operands of each storage type.
#pragma once

#include "device.hpp"
#include "internal.h"
#include "mx_device.hpp"

namespace exemcl {

// ---------------------------------------------------------------------------
// Activations.  sigma(z) = 1 / (1 + e^-z); FAST (results of 16 bits): the exponential
// and the reciprocal of the instructions, together within (1.25 |z| + 5) 2^-24 of the
// value, 2^-17.6 at |z| = 64 (the argument's own rounding and its constant's are most of
// it; the six roundings that make gelu_tanh's z add 6 |z| 2^-24, 2^-15 there), against
// the 2^-12 at least of the result's type.
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
// would round to an infinity keeps the largest bf16 as its upper part.  Of an
// infinity that leaves one, whose rest is NaN; a NaN is NaN from the second part on.
// Parts count down to 2^-133, so that values below 2^-110 lose up to 2^-134.
// ---------------------------------------------------------------------------
typedef float f32x8 __attribute__((ext_vector_type(8)));
__device__ __forceinline__ void split_parts(f32x8 x, bf16x8 &hi, bf16x8 &mid, bf16x8 &lo) {
    typedef float pair __attribute__((ext_vector_type(2)));
    typedef __bf16 rounded __attribute__((ext_vector_type(2)));
    constexpr float kMost = 0x1.fefffep+127f;  // rounds to the largest bf16
    uint32_t part[3][4];
    // A dword of two rounded values, and the values without them: one conversion for both.
    auto take = [](pair &v, pair from) {
        const uint32_t bits = __builtin_bit_cast(uint32_t, __builtin_convertvector(from, rounded));
        v -= pair{__uint_as_float(bits << 16), __uint_as_float(bits & 0xffff0000u)};
        return bits;
    };
#pragma unroll
    for (int e = 0; e < 4; ++e) {
        pair v{x[2 * e], x[2 * e + 1]};
        part[0][e] = take(v, pair{__builtin_amdgcn_fmed3f(v[0], -kMost, kMost), __builtin_amdgcn_fmed3f(v[1], -kMost, kMost)});
        part[1][e] = take(v, v);
        part[2][e] = take(v, v);
    }
    hi = __builtin_bit_cast(bf16x8, part[0]);
    mid = __builtin_bit_cast(bf16x8, part[1]);
    lo = __builtin_bit_cast(bf16x8, part[2]);
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
