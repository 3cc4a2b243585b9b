// mx_device.hpp -- microscaled rows: 8- and 4-bit floating-point elements
// with one power-of-two scale per 32 coordinates (the OCP microscaling
// formats MXFP8 E4M3 and MXFP4 E2M1).
//
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

#include "device.hpp"
#include "mx_layout.hpp"

namespace exemcl {

// ---------------------------------------------------------------------------
// Rounding of one block.  With the largest magnitude 2^e (1 + f), the scale is
// 2^(e - emax), emax the exponent of the element type's largest power of two
// (2 and 8): every element is below 2^(emax + 1) in units of it, is rounded
// to nearest (ties to even) and ends at the largest value (6 and 448).
// ---------------------------------------------------------------------------
// The scale byte, from the largest magnitude's bits: an infinity or a NaN
// anywhere in the block makes it 255.
template <int BITS>
__device__ __forceinline__ uint32_t mx_scale_of(uint32_t amax_bits) {
    constexpr int emax = BITS == 4 ? 2 : 8;
    const int e = (int)(amax_bits >> 23);
    return e == 255 ? 255u : (uint32_t)max(e - emax, 0);
}

// 2^-(scale - 127), what the block is multiplied by (scale <= 252).
__device__ __forceinline__ float mx_inverse(uint32_t scale) { return __uint_as_float((254u - scale) << 23); }

// 2^(scale - 127).
__device__ __forceinline__ float mx_factor(uint32_t scale) {
    return __uint_as_float(scale == 255 ? 0x7fc00000u : scale == 0 ? 0x00400000u : scale << 23);
}

// Eight elements, already in units of the scale, as codes: a dword of 4-bit
// ones (in .x) or two of 8-bit ones.
typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));
typedef short i16x2 __attribute__((ext_vector_type(2)));
typedef float f32x2 __attribute__((ext_vector_type(2)));

template <int BITS>
__device__ __forceinline__ u32x2 mx_encode8(const float (&v)[8]) {
    if constexpr (BITS == 4) {
        // (the conversion ends at 6 by itself)
        uint32_t c = 0;
        c = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(c, v[0], v[1], 1.0f, 0);
        c = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(c, v[2], v[3], 1.0f, 1);
        c = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(c, v[4], v[5], 1.0f, 2);
        c = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(c, v[6], v[7], 1.0f, 3);
        return u32x2{c, 0};
    } else {
        // (past 464 the conversion gives NaN)
        float w[8];
#pragma unroll
        for (int i = 0; i < 8; ++i) w[i] = __builtin_amdgcn_fmed3f(v[i], -448.0f, 448.0f);
        uint32_t a = 0, b = 0;
        a = __builtin_amdgcn_cvt_pk_fp8_f32(w[0], w[1], a, false);
        a = __builtin_amdgcn_cvt_pk_fp8_f32(w[2], w[3], a, true);
        b = __builtin_amdgcn_cvt_pk_fp8_f32(w[4], w[5], b, false);
        b = __builtin_amdgcn_cvt_pk_fp8_f32(w[6], w[7], b, true);
        return u32x2{a, b};
    }
}

template <int BITS>
__device__ __forceinline__ void mx_decode8(u32x2 c, float (&v)[8]) {
    f32x2 p[4];
    if constexpr (BITS == 4) {
        p[0] = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(c.x, 1.0f, 0);
        p[1] = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(c.x, 1.0f, 1);
        p[2] = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(c.x, 1.0f, 2);
        p[3] = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(c.x, 1.0f, 3);
    } else {
        p[0] = __builtin_amdgcn_cvt_pk_f32_fp8((int)c.x, false);
        p[1] = __builtin_amdgcn_cvt_pk_f32_fp8((int)c.x, true);
        p[2] = __builtin_amdgcn_cvt_pk_f32_fp8((int)c.y, false);
        p[3] = __builtin_amdgcn_cvt_pk_f32_fp8((int)c.y, true);
    }
#pragma unroll
    for (int i = 0; i < 8; ++i) v[i] = p[i / 2][i % 2];
}

// The largest of four consecutive lanes' values (the lanes of one block).
__device__ __forceinline__ uint32_t quad_max(uint32_t x) {
    x = max(x, (uint32_t)__builtin_amdgcn_mov_dpp((int)x, 0xb1, 0xf, 0xf, true));  // lanes 1 0 3 2
    x = max(x, (uint32_t)__builtin_amdgcn_mov_dpp((int)x, 0x4e, 0xf, 0xf, true));  // lanes 2 3 0 1
    return x;
}

// Rounds and stores the 8 coordinates c * 8 ... of a row; lanes 4q .. 4q + 3
// hold consecutive chunks of one block and are all active.  `store` false:
// nothing is written.
template <int BITS>
__device__ __forceinline__ void mx_store8(const float (&y)[8], bool store, uint8_t *codes, uint8_t *scales, int c) {
    uint32_t big = 0;
#pragma unroll
    for (int i = 0; i < 8; ++i) big = max(big, __float_as_uint(y[i]) & 0x7fffffffu);
    const uint32_t scale = mx_scale_of<BITS>(quad_max(big));
    const float inv = mx_inverse(min(scale, 253u));
    float v[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) v[i] = y[i] * inv;
    const u32x2 code = mx_encode8<BITS>(v);
    if (!store) return;
    if constexpr (BITS == 4)
        *reinterpret_cast<uint32_t *>(codes + (int64_t)c * 4) = code.x;
    else
        *reinterpret_cast<u32x2 *>(codes + (int64_t)c * 8) = code;
    if ((c & 3) == 0) scales[c >> 2] = (uint8_t)scale;
}

// ---------------------------------------------------------------------------
// Eight consecutive elements of a row; `have` of them are inside it (the
// others read as zeros and are not written).  Rows need no alignment beyond
// their element's.
// ---------------------------------------------------------------------------
template <typename T>
struct Chunk {
    typedef T vec __attribute__((ext_vector_type(8), aligned(sizeof(T))));
};

// ONCE: read once and past the caches, whose room is for what is read again.
template <bool ONCE = false, typename T>
__device__ __forceinline__ typename Chunk<T>::vec load8(const T *p, int have) {
    if (have >= 8) {
        const auto *at = reinterpret_cast<const typename Chunk<T>::vec *>(p);
        if constexpr (ONCE) return __builtin_nontemporal_load(at);
        return *at;
    }
    typename Chunk<T>::vec x;
#pragma unroll
    for (int i = 0; i < 8; ++i) x[i] = i < have ? p[i] : (T)0.0f;
    return x;
}

template <bool ONCE = false, typename T>
__device__ __forceinline__ void load8(const T *p, int have, float (&v)[8]) {
    const auto x = load8<ONCE>(p, have);
#pragma unroll
    for (int i = 0; i < 8; ++i) v[i] = to_f32((T)x[i]);
}

// STREAM: past the caches, which the array does not fit.
template <typename T, bool STREAM = false>
__device__ __forceinline__ void store8(T *p, int have, const float (&v)[8]) {
    if (have >= 8) {
        typename Chunk<T>::vec x;
#pragma unroll
        for (int i = 0; i < 8; ++i) x[i] = (T)v[i];
        if constexpr (STREAM)
            __builtin_nontemporal_store(x, reinterpret_cast<typename Chunk<T>::vec *>(p));
        else
            *reinterpret_cast<typename Chunk<T>::vec *>(p) = x;
    } else {
#pragma unroll
        for (int i = 0; i < 8; ++i)
            if (i < have) p[i] = (T)v[i];
    }
}

// ---------------------------------------------------------------------------
// Matrix-core operands.  One 16x16x128 instruction: lane L holds row
// L % 16 of its operand and belongs to K-group g = L / 16.
//   4 bits  coordinates 32 g .. 32 g + 31: 16 consecutive bytes of the row
//   8 bits  coordinates 16 g .. 16 g + 15 and 64 + 16 g .. 64 + 16 g + 15
//   scale   of coordinates 32 g .. 32 g + 31, either way
// Results: accumulator i of a lane is row 4 g + i of the first operand and
// row L % 16 of the second.
// ---------------------------------------------------------------------------
typedef int i32x4 __attribute__((ext_vector_type(4)));
typedef int i32x8 __attribute__((ext_vector_type(8)));

__device__ __forceinline__ i32x8 mx_wide(i32x8 x) { return x; }
__device__ __forceinline__ i32x8 mx_wide(i32x4 x) { return __builtin_shufflevector(x, x, 0, 1, 2, 3, -1, -1, -1, -1); }
__device__ __forceinline__ i32x8 mx_join(i32x4 lo, i32x4 hi) {
    return i32x8{lo[0], lo[1], lo[2], lo[3], hi[0], hi[1], hi[2], hi[3]};
}

// a and b: i32x4 of 4-bit elements, i32x8 of 8-bit ones; SEL: the byte of the
// scale operand that counts.
template <int SEL_A = 0, int SEL_B = 0, typename A, typename B>
__device__ __forceinline__ f32x4 mx_mma(A a, B b, f32x4 c, int scale_a, int scale_b) {
    return __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(mx_wide(a), mx_wide(b), c, sizeof(A) == 16 ? 4 : 0,
                                                            sizeof(B) == 16 ? 4 : 0, SEL_A, scale_a, SEL_B, scale_b);
}

// x = high + low, element by element: the 8-bit codes of magnitude >= 2 and
// the others.  The instruction adds the products of 8 consecutive coordinates
// with 13 bits below the largest sum of two exponents.  Those of 8-bit elements
// are -6 .. 8, of 4-bit ones 0 .. 2, and a product has 4 bits below their sum: up
// to 20 binades in all, but 13 among the large elements and 12 among the others.
// So each part's sum is exact.  Results of 16 bits need it like those of 32: not
// divided, 448 and -448 beside six elements of 0.015 leave nothing of these, and
// with one element per 8 a hundred times the others one result in ten is off by
// more than half a step of fp16.
__device__ __forceinline__ void mx_divide(i32x8 x, i32x8 &high, i32x8 &low) {
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        const uint32_t t = (uint32_t)x[i] & 0x40404040u, m = (t << 1) - (t >> 6);  // 7f where it is set
        high[i] = x[i] & (int)(m | 0x80808080u);
        low[i] = x[i] & (int)~m;
    }
}

}  // namespace exemcl
