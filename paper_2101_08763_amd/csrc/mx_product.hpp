// mx_product.hpp -- products of microscaled rows, A (8 or 4 bits) with B (4
// bits): C[i][j] = sum_t A[i][t] B[j][t] + bias[j] (instantiated in
// kernels_mx_product_*.hip, one per format of A).
#pragma once

#include "internal.h"
#include "mfma_kernels.hpp"
#include "mx_device.hpp"

namespace exemcl {

// A 16 x 16 tile of C per workgroup, operands from memory; the K-steps of 128
// coordinates go to the wavefronts in turn, whose sums are added in order.
constexpr int kDirectWaves = 4;

template <typename T, int BITS_A, bool DIVIDE>
__global__ __launch_bounds__(kDirectWaves * 64) void mx_product_direct_kernel(
    const uint8_t *__restrict__ A, const uint8_t *__restrict__ As, int64_t m, const uint8_t *__restrict__ B,
    const uint8_t *__restrict__ Bs, int64_t n, int64_t d, int64_t ntiles, const float *__restrict__ bias,
    T *__restrict__ C) {
    __shared__ f32x4 sums[kDirectWaves][64];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, lr = lane & 15, g = lane >> 4;
    const int64_t unit = flat_block(), mt = unit / ntiles, nt = unit - mt * ntiles;
    if (mt * 16 >= m) return;
    const int64_t ar = min(mt * 16 + lr, m - 1), br = min(nt * 16 + lr, n - 1);
    const uint8_t *a_row = A + ar * mx_row_bytes(d, BITS_A), *as_row = As + ar * mx_row_scales(d);
    const uint8_t *b_row = B + br * mx_row_bytes(d, 4), *bs_row = Bs + br * mx_row_scales(d);
    const int ksteps = (int)(mx_padded(d) / kMxRow);
    f32x4 acc = {0.0f, 0.0f, 0.0f, 0.0f};
    for (int ks = wave; ks < ksteps; ks += kDirectWaves) {
        const i32x4 b = *reinterpret_cast<const i32x4 *>(b_row + ks * 64 + g * 16);
        const int sa = as_row[ks * 4 + g], sb = bs_row[ks * 4 + g];
        if constexpr (BITS_A == 4) {
            acc = mx_mma(b, *reinterpret_cast<const i32x4 *>(a_row + ks * 64 + g * 16), acc, sb, sa);
        } else {
            const i32x8 a = mx_join(*reinterpret_cast<const i32x4 *>(a_row + ks * 128 + g * 16),
                                    *reinterpret_cast<const i32x4 *>(a_row + ks * 128 + 64 + g * 16));
            if constexpr (DIVIDE) {
                i32x8 high, low;
                mx_divide(a, high, low);
                acc = mx_mma(b, low, acc, sb, sa);
                acc = mx_mma(b, high, acc, sb, sa);
            } else {
                acc = mx_mma(b, a, acc, sb, sa);
            }
        }
    }
    sums[wave][lane] = acc;
    __syncthreads();
    if (wave != 0) return;
#pragma unroll
    for (int w = 1; w < kDirectWaves; ++w) acc += sums[w][lane];
    const int64_t row = mt * 16 + lr;
    if (row >= m) return;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const int64_t col = nt * 16 + 4 * g + i;
        if (col < n) C[row * n + col] = (T)(bias ? acc[i] + bias[col] : acc[i]);
    }
}

template <typename T, int BITS_A, bool DIVIDE>
hipError_t product_launch(const MxProductArgs &a, hipStream_t st) {
    const int64_t mt = (a.m + 15) / 16, nt = (a.n + 15) / 16;
    if (mt > (int64_t(1) << 34) / nt) return hipErrorInvalidValue;  // 2^14 rows of kFlatRow
    hipLaunchKernelGGL((mx_product_direct_kernel<T, BITS_A, DIVIDE>), flat_grid(mt * nt, kDirectWaves * 64),
                       dim3(kDirectWaves * 64), 0, st, (const uint8_t *)a.A, (const uint8_t *)a.A_scales, a.m,
                       (const uint8_t *)a.B, (const uint8_t *)a.B_scales, a.n, a.d, nt, a.bias, (T *)a.C);
    return hipGetLastError();
}

// DIVIDE: 8-bit rows in two parts (mx_divide), for results in fp32; what the
// matrix cores drop otherwise is far below the rounding of a 16-bit result.
template <int BITS_A>
hipError_t product_typed(int prec, const MxProductArgs &a, hipStream_t st) {
    if (prec == P_FP32) return product_launch<float, BITS_A, BITS_A == 8>(a, st);
    if (prec == P_FP16) return product_launch<_Float16, BITS_A, false>(a, st);
    return product_launch<__bf16, BITS_A, false>(a, st);
}

}  // namespace exemcl
