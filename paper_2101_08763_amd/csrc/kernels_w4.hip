// kernels_w4.hip -- making and unmaking weights of 4 bits with group scales, one
// pass over memory each (exemcl.h has the rule, w4_layout.hpp the order).
#include <algorithm>

#include "w4_rows.hpp"

namespace exemcl {

namespace {

// The largest number of a type.
template <typename T>
constexpr float kLargest = 0x1.fffffep127f;
template <>
constexpr float kLargest<_Float16> = 65504.0f;
template <>
constexpr float kLargest<__bf16> = 0x1.fep127f;

// A wavefront takes a tile of 16 rows x 128 coordinates: lane (r, q) row r and the
// coordinates 32 j + 8 q + e, which are its 16 bytes.  A group's extremes are those
// of the lanes q of a row, over the j that belong to it.  HBM-bound: 32 768 rows of
// 8 192 of bf16 by groups of 128 124 us (5.5 TB/s), of fp32 217 (5.6), by groups of 32, with
// four divisions for one, 137 and 228 (5.1, 5.4); 8 192 x 4 096 of bf16 20 and 23 (4.3, 3.8).
template <typename T, int GROUP>
__global__ __launch_bounds__(256) void w4_quantize_kernel(const T *__restrict__ w, int64_t n, int64_t d, int64_t units,
                                                          u32x4 *__restrict__ codes, uint32_t *__restrict__ words) {
    constexpr int STEPS = GROUP / 32, GPB = 4 / STEPS;
    const int lane = threadIdx.x & 63, r = lane & 15, q = lane >> 4;
    const int64_t unit = flat_block() * 4 + (threadIdx.x >> 6), blocks = w4_blocks(d);
    if (unit >= units) return;
    const int64_t tile = unit / blocks, b = unit - tile * blocks, row = tile * 16 + r;
    float v[4][8];
#pragma unroll
    for (int j = 0; j < 4; ++j) {
        const int64_t k = b * kW4Block + 32 * j + 8 * q;
        const bool in = row < n && k < d;
        load8<true>(w + (in ? row * d + k : 0), in ? (int)min((int64_t)8, d - k) : 0, v[j]);
    }
    u32x4 out;
#pragma unroll
    for (int p = 0; p < GPB; ++p) {
        float lo = 0.0f, hi = 0.0f, odd = 0.0f;  // odd: NaN where a value is not finite
#pragma unroll
        for (int j = p * STEPS; j < (p + 1) * STEPS; ++j)
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                lo = fminf(lo, v[j][e]);
                hi = fmaxf(hi, v[j][e]);
                odd += v[j][e] * 0.0f;
            }
#pragma unroll
        for (int off = 16; off <= 32; off <<= 1) {
            lo = fminf(lo, __shfl_xor(lo, off));
            hi = fmaxf(hi, __shfl_xor(hi, off));
            odd += __shfl_xor(odd, off);
        }
        // (halves: the range may pass the largest number; a scale without a
        // reciprocal counts as 0)
        const float s0 = (hi * 0.5f - lo * 0.5f) / 7.5f;
        const bool bad = odd != odd;
        const uint32_t sbits = bad ? 0x7fc00000u : s0 < 0x1p-126f ? 0u : (__float_as_uint(s0) + 255u) & ~255u;
        const float s = __uint_as_float(sbits), inv = s > 0.0f ? 1.0f / s : 0.0f;
        const float z = bad ? 0.0f : fminf(fmaxf(rintf(-lo * inv), 0.0f), 15.0f);
        // Where a value of the group may round to an infinity, a code whose value does goes
        // one step towards z: that is enough, it is half a step at most past its weight.
        const bool far = s * 15.0f > kLargest<T>;
#pragma unroll
        for (int j = p * STEPS; j < (p + 1) * STEPS; ++j) {
            uint32_t c = 0;
            float t[8];
#pragma unroll
            for (int e = 0; e < 8; ++e) t[e] = fminf(fmaxf(rintf(v[j][e] * inv) + z, 0.0f), 15.0f);
            if (__builtin_amdgcn_ballot_w64(far) != 0)  // (a jump over it)
#pragma unroll
                for (int e = 0; e < 8; ++e)
                    if (__builtin_isinf(to_f32((T)((t[e] - z) * s)))) t[e] += t[e] > z ? -1.0f : 1.0f;
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                const int64_t k = b * kW4Block + 32 * j + 8 * q + e;
                const uint32_t code = bad || row >= n || k >= d ? 0u : (uint32_t)t[e];
                c |= code << (e % 4 * 8 + e / 4 * 4);
            }
            out[j] = c;
        }
        if (q == 0) words[(tile * blocks * GPB + b * GPB + p) * 16 + r] = sbits | (uint32_t)z;
    }
    codes[unit * 64 + lane] = out;
}

// A wavefront takes a tile, and each of its stores whole rows of it, 16 bytes a lane:
// a lane's values are half a dword of codes (fp32) or a whole one.  HBM-bound: 32 768
// rows of 4 096 to bf16 52 us (6.5 TB/s), to fp32 108 (5.6); rows of 8 192 to bf16 124 (5.5),
// to fp32, more than 0.8 GB of it, 290 (4.2).  Lanes that take the 16
// bytes of codes in quantize's order store 64 bytes of a row at a time: 59 and, past
// the caches, 247 us.
template <typename T, bool STREAM>
__global__ __launch_bounds__(256) void w4_dequantize_kernel(const uint32_t *__restrict__ codes,
                                                            const uint32_t *__restrict__ words, int64_t n, int64_t d,
                                                            int steps, int64_t units, T *__restrict__ w) {
    constexpr int PER = 16 / sizeof(T), LANES = kW4Block / PER, ROWS = 64 / LANES;  // ROWS at a time
    typedef T vec __attribute__((ext_vector_type(PER), aligned(sizeof(T))));
    const int lane = threadIdx.x & 63, at = lane % LANES * PER;
    const int64_t unit = flat_block() * 4 + (threadIdx.x >> 6), blocks = w4_blocks(d);
    if (unit >= units) return;
    const int64_t tile = unit / blocks, b = unit - tile * blocks, k = b * kW4Block + at;
    if (k >= d) return;
    const int have = (int)min((int64_t)PER, d - k), j = at / 32, p = at % 32 / 8;
    const uint32_t shift = at % 8;  // 0, or 4 for the high halves
    const uint32_t *code = codes + unit * 256 + 64 * p + j, *word = words + (unit * (4 / steps) + j / steps) * 16;
#pragma unroll
    for (int i = 0; i < 16 / ROWS; ++i) {
        const int r = i * ROWS + lane / LANES;
        const int64_t row = tile * 16 + r;
        if (row >= n) return;
        const uint32_t c = code[4 * r] >> shift, sz = word[r];
        const float s = __uint_as_float(sz & 0xffffff00u), z = (float)(sz & 0xffu);
        vec x;
#pragma unroll
        for (int e = 0; e < PER; ++e) x[e] = (T)(((float)(c >> (e % 4 * 8 + e / 4 * 4) & 15u) - z) * s);
        T *to = w + row * d + k;
        if (have < PER) {
#pragma unroll
            for (int e = 0; e < PER - 1; ++e)
                if (e < have) to[e] = x[e];
        } else if constexpr (STREAM) {
            __builtin_nontemporal_store(x, reinterpret_cast<vec *>(to));
        } else {
            *reinterpret_cast<vec *>(to) = x;
        }
    }
}

template <typename T>
hipError_t quantize(const void *w, int64_t n, int64_t d, int group, void *codes, void *words, hipStream_t st) {
    const int64_t units = w4_tiles(n) * w4_blocks(d);
    if (units > int64_t(1) << 35) return hipErrorInvalidValue;
    auto go = [&](auto kern) {
        hipLaunchKernelGGL(kern, flat_grid((units + 3) / 4, 256), dim3(256), 0, st, (const T *)w, n, d, units,
                           (u32x4 *)codes, (uint32_t *)words);
    };
    if (group == 32)
        go(w4_quantize_kernel<T, 32>);
    else if (group == 64)
        go(w4_quantize_kernel<T, 64>);
    else
        go(w4_quantize_kernel<T, 128>);
    return hipGetLastError();
}

// Values that fill half the last-level cache (256 MiB) or more are stored past it (us,
// through it and past it: 134 MB of fp32 38 / 26, of bf16 35 / 26, 537 MB 149 / 107 and
// 126 / 124, 1.07 GB 300 / 290 and 248 / 242; 541 MB of bf16 rows of odd length 198 / 214).
// Fewer may be read from it next.
constexpr int64_t kStreamBytes = int64_t(128) << 20;

template <typename T>
hipError_t dequantize(const void *codes, const void *words, int64_t n, int64_t d, int group, void *w, hipStream_t st) {
    const int64_t units = w4_tiles(n) * w4_blocks(d);
    if (units > int64_t(1) << 35) return hipErrorInvalidValue;
    auto go = [&](auto kern) {
        hipLaunchKernelGGL(kern, flat_grid((units + 3) / 4, 256), dim3(256), 0, st, (const uint32_t *)codes,
                           (const uint32_t *)words, n, d, group / 32, units, (T *)w);
    };
    if (n * d * (int64_t)sizeof(T) >= kStreamBytes)
        go(w4_dequantize_kernel<T, true>);
    else
        go(w4_dequantize_kernel<T, false>);
    return hipGetLastError();
}

}  // namespace

hipError_t launch_w4_quantize(int prec, const void *w, int64_t n, int64_t d, int group, void *codes, void *words,
                              hipStream_t st) {
    if (n == 0) return hipSuccess;
    if (prec == P_FP32) return quantize<float>(w, n, d, group, codes, words, st);
    if (prec == P_FP16) return quantize<_Float16>(w, n, d, group, codes, words, st);
    return quantize<__bf16>(w, n, d, group, codes, words, st);
}

hipError_t launch_w4_dequantize(int prec, const void *codes, const void *words, int64_t n, int64_t d, int group, void *w,
                                hipStream_t st) {
    if (n == 0) return hipSuccess;
    if (prec == P_FP32) return dequantize<float>(codes, words, n, d, group, w, st);
    if (prec == P_FP16) return dequantize<_Float16>(codes, words, n, d, group, w, st);
    return dequantize<__bf16>(codes, words, n, d, group, w, st);
}

hipError_t launch_w4_rows(int prec, const W4Args &a, hipStream_t st) {
    if (prec == P_FP32) return w4_run_f32(a, st);
    if (prec == P_FP16) return w4_run_f16(a, st);
    return w4_run_bf16(a, st);
}

}  // namespace exemcl
