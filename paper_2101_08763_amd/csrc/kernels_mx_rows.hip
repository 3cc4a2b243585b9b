// kernels_mx_rows.hip -- what makes and unmakes microscaled rows, one pass
// over memory each: rounding, its inverse, and the root-mean-square norm with
// the residual's addition and its gradient.
#include <algorithm>

#include "internal.h"
#include "mfma_kernels.hpp"
#include "mx_device.hpp"

namespace exemcl {

namespace {

// Quotients by a number fixed for the launch, of dividends below 2^31.
struct Divider {
    uint32_t mul, shift, by;
};
Divider divider(uint32_t by) {
    uint32_t s = 0;
    while ((1ull << s) < by) ++s;
    return {(uint32_t)(((1ull << 32) * ((1ull << s) - by)) / by + 1), s, by};
}
__device__ __forceinline__ uint32_t divide(uint32_t x, Divider d) { return (__umulhi(x, d.mul) + x) >> d.shift; }

// Launches with at most this many 8-coordinate chunks.
constexpr int64_t kMaxChunks = int64_t(1) << 30;

// ---------------------------------------------------------------------------
// Rounding.  A lane takes 8 coordinates, four lanes a block.  HBM-bound: 10^6 x
// 256 fp16 to 4 bits in 112 us (5.8 TB/s) and back in 93 (7.0).
// ---------------------------------------------------------------------------
template <typename T, int BITS>
__global__ __launch_bounds__(256) void mx_quantize_kernel(const T *__restrict__ x, uint32_t chunks, Divider per_row,
                                                          int d, uint8_t *__restrict__ codes,
                                                          uint8_t *__restrict__ scales) {
    const uint32_t i = blockIdx.x * 256u + threadIdx.x, j = min(i, chunks - 1);
    const uint32_t row = divide(j, per_row), c = j - row * per_row.by;
    const int d0 = (int)c * 8;
    float y[8];
    load8<true>(x + (int64_t)row * d + d0, d - d0, y);
    const int64_t rb = (int64_t)per_row.by * BITS, rs = per_row.by / 4;
    mx_store8<BITS>(y, i < chunks, codes + row * rb, scales + row * rs, (int)c);
}

template <typename T, int BITS, bool STREAM>
__global__ __launch_bounds__(256) void mx_dequantize_kernel(const uint8_t *__restrict__ codes,
                                                            const uint8_t *__restrict__ scales, uint32_t chunks,
                                                            Divider per_row, int d, T *__restrict__ x) {
    const uint32_t i = blockIdx.x * 256u + threadIdx.x;
    if (i >= chunks) return;
    const uint32_t row = divide(i, per_row), c = i - row * per_row.by;
    const int64_t rb = mx_row_bytes(d, BITS), rs = mx_row_scales(d);
    u32x2 code = {0, 0};
    if constexpr (BITS == 4)
        code.x = *reinterpret_cast<const uint32_t *>(codes + row * rb + c * 4);
    else
        code = *reinterpret_cast<const u32x2 *>(codes + row * rb + c * 8);
    const float f = mx_factor(scales[row * rs + c / 4]);
    float v[8];
    mx_decode8<BITS>(code, v);
#pragma unroll
    for (int e = 0; e < 8; ++e) v[e] *= f;
    const int d0 = (int)c * 8;
    store8<T, STREAM>(x + (int64_t)row * d + d0, d - d0, v);
}

// ---------------------------------------------------------------------------
// Root-mean-square norm:  v = x + r,  y = v w / sqrt(mean(v^2) + eps).
//
// TPR threads share a row, chunk t + i TPR of 8 coordinates going to thread t;
// the row stays in registers (CPT chunks a thread) between the sum of squares
// and the result.  CPT = 0: rows too long for that, read twice.  HBM-bound:
// 20 000 x 1 536 bf16 with a residual to 8 bits in 40 us (5.3 TB/s; 45 when x and r
// are kept in the caches, which then hold less of what is written).
//
// The sum and its root are held in 64 bits, and on the way to 8 or 4 bits y in
// two parts, rounded to odd: a row's last bit decides on which side of a power of
// two a block's maximum falls, and with it the whole block's scale, and rounding
// to 24 bits first would make ties of what are none (of 31 million codes 20 came
// out wrong).  The second part takes 2 us of these 40.
// ---------------------------------------------------------------------------
template <int TPR, typename S>
__device__ __forceinline__ S row_sum(S s, S *lds) {
#pragma unroll
    for (int off = min(TPR, 64) / 2; off >= 1; off >>= 1) s += __shfl_xor(s, off);
    if constexpr (TPR > 64) {
        __syncthreads();  // the last row's sums have been read
        if ((threadIdx.x & 63) == 0) lds[threadIdx.x >> 6] = s;
        __syncthreads();
        s = 0;
#pragma unroll
        for (int w = 0; w < TPR / 64; ++w) s += lds[w];
    }
    return s;
}

// 1 / sqrt(m): the instruction's 26 bits and one step of Newton's iteration.  Its
// ends (m = 0, infinite, NaN) are the instruction's own.
__device__ __forceinline__ double inverse_root(double m) {
    const double r = __builtin_amdgcn_rsq(m), half = 0.5 * r;
    const double t = fma(fma(-m * r, r, 1.0), half, r);
    return r > 0.0 && r < (double)INFINITY ? t : r;
}

// y0 + rest in 24 bits that are rounded again later: where y0 is not all of it,
// the neighbour with an odd last bit, which no midpoint of fewer bits has.  Of a y0
// that is infinite the rest is too, or NaN, and it stays.
__device__ __forceinline__ float to_odd(float y0, float rest) {
    const int b = __float_as_int(y0), step = (b ^ __float_as_int(rest)) >> 31 | 1;
    constexpr int finite = 0x198;  // normal or subnormal, of either sign
    return __builtin_amdgcn_classf(rest, finite) && (b & 1) == 0 && b << 1 != 0 ? __int_as_float(b + step) : y0;
}

constexpr int norm_block(int tpr) { return tpr > 256 ? tpr : 256; }

template <typename T, int BITS, int TPR, int CPT>
__global__ __launch_bounds__(norm_block(TPR)) void rmsnorm_kernel(const T *x, const T *r,
                                                                  const T *__restrict__ w, int64_t n, int d,
                                                                  double inv_d, float eps, T *h, T *__restrict__ y, uint8_t *__restrict__ codes,
                                                                  uint8_t *__restrict__ scales,
                                                                  float *__restrict__ rstd_out) {
    constexpr int RPB = norm_block(TPR) / TPR;
    __shared__ double lds[TPR / 64 + 1];
    const int t = threadIdx.x % TPR;
    const int64_t row = flat_block() * RPB + threadIdx.x / TPR;
    const bool live = row < n;
    const int64_t at = (live ? row : n - 1) * d;
    const int chunks = BITS ? (int)(mx_padded(d) / 8) : (d + 7) / 8;
    auto load = [&](int c, float(&v)[8]) {
        const int d0 = c * 8;
        load8<(CPT > 0)>(x + at + d0, d - d0, v);
        if (r) {
            float u[8];
            load8<(CPT > 0)>(r + at + d0, d - d0, u);
#pragma unroll
            for (int e = 0; e < 8; ++e) v[e] += u[e];
        }
    };
    auto finish = [&](int c, const float(&v)[8], float rstd, float low) {
        const int d0 = c * 8;
        if (h && live) store8(h + at + d0, d - d0, v);
        float g[8];
        if (w)
            load8(w + d0, d - d0, g);
        else
#pragma unroll
            for (int e = 0; e < 8; ++e) g[e] = 1.0f;
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            const float p = v[e] * rstd;
            if constexpr (BITS != 0) {
                const float rest = fmaf(v[e], low, fmaf(v[e], rstd, -p)) * g[e], y0 = fmaf(p, g[e], rest);
                g[e] = to_odd(y0, fmaf(p, g[e], -y0) + rest);
            } else {
                g[e] *= p;
            }
        }
        if constexpr (BITS != 0) {
            if (d - d0 < 8)  // past d: zeros, where 0 rstd is not
#pragma unroll
                for (int e = 0; e < 8; ++e) g[e] = e < d - d0 ? g[e] : 0.0f;
            mx_store8<BITS>(g, live && c < chunks, codes + row * mx_row_bytes(d, BITS), scales + row * mx_row_scales(d), c);
        } else if (live) {
            store8(y + at + d0, d - d0, g);
        }
    };
    double s = 0.0;
    if constexpr (CPT > 0) {
        float v[CPT][8];
#pragma unroll
        for (int i = 0; i < CPT; ++i) {
            load(t + i * TPR, v[i]);
#pragma unroll
            for (int e = 0; e < 8; ++e) s = fma((double)v[i][e], (double)v[i][e], s);
        }
        s = inverse_root(row_sum<TPR>(s, lds) * inv_d + (double)eps);
        const float rstd = (float)s, low = (float)(s - rstd);
#pragma unroll
        for (int i = 0; i < CPT; ++i) finish(t + i * TPR, v[i], rstd, low);
    } else {
        for (int c = t; c < chunks; c += TPR) {
            float v[8];
            load(c, v);
#pragma unroll
            for (int e = 0; e < 8; ++e) s = fma((double)v[e], (double)v[e], s);
        }
        s = inverse_root(row_sum<TPR>(s, lds) * inv_d + (double)eps);
        const float rstd = (float)s, low = (float)(s - rstd);
        // whole blocks of four lanes take every step together (chunks is a
        // multiple of 4 where it matters)
        for (int c = t; c < chunks; c += TPR) {
            float v[8];
            load(c, v);
            finish(c, v, rstd, low);
        }
    }
    if (rstd_out && live && t == 0) rstd_out[row] = (float)s;
}

// ---------------------------------------------------------------------------
// Its gradient, from the saved v = h and rstd:  with xhat = h rstd and
// g = dy w,  dx = rstd (g - xhat mean(g xhat)) + dh  and  dw = sum over rows
// of dy xhat.  A thread keeps the same columns for all rows it sees, their
// weights and their part of dw in registers, and loads a row while it works on
// the one before; a workgroup's parts are added in LDS in a
// fixed order and written as one row of `partial` (grid x d).  HBM-bound: 20 000 x
// 1 536 bf16 in 42 us (5.9 TB/s), and 4.6 for the sum of 512 parts; 47 and 4.6
// when the rows are kept in the caches.
// ---------------------------------------------------------------------------
template <typename T, int TPR, int CPT>
__global__ __launch_bounds__(256) void rmsnorm_grad_kernel(const T *__restrict__ dy, const T *__restrict__ h,
                                                           const T *__restrict__ w, const float *__restrict__ rstd_in,
                                                           const T *__restrict__ dh, int64_t n, int d,
                                                           T *__restrict__ dx, float *__restrict__ partial) {
    using vec = typename Chunk<T>::vec;
    constexpr int RPB = 256 / TPR, COLS = TPR * CPT * 8;
    __shared__ float lds[8];
    __shared__ float sums[RPB > 1 ? RPB * COLS : 1];
    const int t = threadIdx.x % TPR, slot = threadIdx.x / TPR;
    float dw[CPT][8] = {};
    vec ww[CPT], nh[CPT], ng[CPT], no[CPT];
    auto load = [&](int64_t row) {
        const int64_t at = min(row, n - 1) * d;
#pragma unroll
        for (int i = 0; i < CPT; ++i) {
            const int d0 = (t + i * TPR) * 8;
            nh[i] = load8<true>(h + at + d0, d - d0);
            ng[i] = load8<true>(dy + at + d0, d - d0);
            if (dh) no[i] = load8<true>(dh + at + d0, d - d0);
        }
    };
#pragma unroll
    for (int i = 0; i < CPT; ++i) {
        const int d0 = (t + i * TPR) * 8;
        if (w)
            ww[i] = load8(w + d0, d - d0);
        else
#pragma unroll
            for (int e = 0; e < 8; ++e) ww[i][e] = (T)1.0f;
    }
    load((int64_t)blockIdx.x * RPB + slot);
    for (int64_t base = (int64_t)blockIdx.x * RPB; base < n; base += (int64_t)gridDim.x * RPB) {
        const int64_t row = base + slot;
        const bool live = row < n;
        const float rstd = rstd_in[live ? row : n - 1];
        vec ch[CPT], cg[CPT], co[CPT];
#pragma unroll
        for (int i = 0; i < CPT; ++i) ch[i] = nh[i], cg[i] = ng[i], co[i] = no[i];
        load(row + (int64_t)gridDim.x * RPB);  // the next row's, or the last one again
        float s = 0.0f;
#pragma unroll
        for (int i = 0; i < CPT; ++i)
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                const float xh = to_f32((T)ch[i][e]) * rstd, g = to_f32((T)cg[i][e]);
                if (live) dw[i][e] = fmaf(g, xh, dw[i][e]);
                s = fmaf(g * to_f32((T)ww[i][e]), xh, s);
            }
        const float c = row_sum<TPR>(s, lds) / (float)d;
#pragma unroll
        for (int i = 0; i < CPT; ++i) {
            const int d0 = (t + i * TPR) * 8;
            float o[8];
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                const float xh = to_f32((T)ch[i][e]) * rstd, g = to_f32((T)cg[i][e]) * to_f32((T)ww[i][e]);
                o[e] = fmaf(rstd, fmaf(-xh, c, g), dh ? to_f32((T)co[i][e]) : 0.0f);
            }
            if (live) store8(dx + (row * d + d0), d - d0, o);
        }
    }
    if (!partial) return;
    float *mine = partial + (int64_t)blockIdx.x * d;
    if constexpr (RPB > 1) {
#pragma unroll
        for (int i = 0; i < CPT; ++i)
#pragma unroll
            for (int e = 0; e < 8; ++e) sums[slot * COLS + (t + i * TPR) * 8 + e] = dw[i][e];
        __syncthreads();
        for (int c = threadIdx.x; c < d; c += 256) {
            float s = 0.0f;
            for (int q = 0; q < RPB; ++q) s += sums[q * COLS + c];
            mine[c] = s;
        }
    } else {
#pragma unroll
        for (int i = 0; i < CPT; ++i) store8(mine + (t + i * TPR) * 8, d - (t + i * TPR) * 8, dw[i]);
    }
}

// Rows too long for registers: dx row by row, read twice, and dw column by
// column, a thread to each, over a block of rows.
template <typename T>
__global__ __launch_bounds__(1024) void rmsnorm_grad_long_kernel(const T *__restrict__ dy, const T *__restrict__ h,
                                                                 const T *__restrict__ w,
                                                                 const float *__restrict__ rstd_in,
                                                                 const T *__restrict__ dh, int d, T *__restrict__ dx) {
    __shared__ float lds[16];
    const int64_t row = blockIdx.x, at = row * d;
    const float rstd = rstd_in[row];
    float s = 0.0f;
    auto load = [&](int d0, float(&xh)[8], float(&g)[8]) {
        load8(h + at + d0, d - d0, xh);
        load8(dy + at + d0, d - d0, g);
        if (w) {
            float ww[8];
            load8(w + d0, d - d0, ww);
#pragma unroll
            for (int e = 0; e < 8; ++e) g[e] *= ww[e];
        }
#pragma unroll
        for (int e = 0; e < 8; ++e) xh[e] *= rstd;
    };
    for (int d0 = threadIdx.x * 8; d0 < d; d0 += 8192) {
        float xh[8], g[8], q = 0.0f;
        load(d0, xh, g);
#pragma unroll
        for (int e = 0; e < 8; ++e) q = fmaf(g[e], xh[e], q);
        s += q;
    }
    const float c = row_sum<1024>(s, lds) / (float)d;
    for (int d0 = threadIdx.x * 8; d0 < d; d0 += 8192) {
        float xh[8], g[8], o[8] = {};
        load(d0, xh, g);
        if (dh) load8(dh + at + d0, d - d0, o);
#pragma unroll
        for (int e = 0; e < 8; ++e) o[e] = fmaf(rstd, fmaf(-xh[e], c, g[e]), o[e]);
        store8(dx + at + d0, d - d0, o);
    }
}

template <typename T>
__global__ __launch_bounds__(256) void rmsnorm_dw_long_kernel(const T *__restrict__ dy, const T *__restrict__ h,
                                                              const float *__restrict__ rstd, int64_t n, int d,
                                                              int64_t rows, float *__restrict__ partial) {
    const int c = blockIdx.x * 256 + threadIdx.x;
    if (c >= d) return;
    const int64_t r0 = blockIdx.y * rows, r1 = min(n, r0 + rows);
    float s = 0.0f;
    for (int64_t r = r0; r < r1; ++r) s = fmaf(to_f32(dy[r * d + c]), to_f32(h[r * d + c]) * rstd[r], s);
    partial[(int64_t)blockIdx.y * d + c] = s;
}

// dw[c] = sum over g of partial[g][c], in 64 bits and a fixed order.
constexpr int kDwCols = 16, kDwRows = 64, kDwUnroll = 8;
__global__ __launch_bounds__(kDwCols *kDwRows) void column_sum_kernel(const float *__restrict__ partial, int G, int d,
                                                                       float *__restrict__ dw) {
    __shared__ double part[kDwRows][kDwCols + 1];
    const int cl = threadIdx.x % kDwCols, q = threadIdx.x / kDwCols, c = blockIdx.x * kDwCols + cl;
    double s = 0.0;
    if (c < d)
        for (int g = q; g < G; g += kDwRows * kDwUnroll) {
            float x[kDwUnroll];
#pragma unroll
            for (int u = 0; u < kDwUnroll; ++u) x[u] = partial[(int64_t)min(g + u * kDwRows, G - 1) * d + c];
#pragma unroll
            for (int u = 0; u < kDwUnroll; ++u) s += g + u * kDwRows < G ? (double)x[u] : 0.0;
        }
    part[q][cl] = s;
    __syncthreads();
#pragma unroll
    for (int w = kDwRows / 2; w >= 1; w >>= 1) {
        if (q < w) part[q][cl] += part[q + w][cl];
        __syncthreads();
    }
    if (q == 0 && c < d) dw[c] = (float)part[0][cl];
}

template <typename T, int BITS>
hipError_t quantize(const void *x, int64_t n, int64_t d, void *codes, void *scales, hipStream_t st) {
    const int64_t per = mx_padded(d) / 8, rows = std::max<int64_t>(1, kMaxChunks / per);
    for (int64_t r = 0; r < n; r += rows) {
        const uint32_t chunks = (uint32_t)(std::min(rows, n - r) * per);
        hipLaunchKernelGGL((mx_quantize_kernel<T, BITS>), dim3((chunks + 255) / 256), dim3(256), 0, st,
                           (const T *)x + r * d, chunks, divider((uint32_t)per), (int)d,
                           (uint8_t *)codes + r * mx_row_bytes(d, BITS), (uint8_t *)scales + r * mx_row_scales(d));
    }
    return hipGetLastError();
}

// Values that do not fit the last-level cache (256 MiB) are stored past it: 512
// MB of fp16 in 93 us instead of 126.  Smaller ones may be read from it next.
constexpr int64_t kStreamBytes = int64_t(256) << 20;

template <typename T, int BITS>
hipError_t dequantize(const void *codes, const void *scales, int64_t n, int64_t d, void *x, hipStream_t st) {
    const auto kern = n * d * (int64_t)sizeof(T) > kStreamBytes ? mx_dequantize_kernel<T, BITS, true>
                                                                : mx_dequantize_kernel<T, BITS, false>;
    const int64_t per = (d + 7) / 8, rows = std::max<int64_t>(1, kMaxChunks / per);
    for (int64_t r = 0; r < n; r += rows) {
        const uint32_t chunks = (uint32_t)(std::min(rows, n - r) * per);
        hipLaunchKernelGGL(kern, dim3((chunks + 255) / 256), dim3(256), 0, st,
                           (const uint8_t *)codes + r * mx_row_bytes(d, BITS),
                           (const uint8_t *)scales + r * mx_row_scales(d), chunks, divider((uint32_t)per), (int)d,
                           (T *)x + r * d);
    }
    return hipGetLastError();
}

template <typename T, int BITS, int TPR, int CPT>
hipError_t norm_launch(const NormArgs &a, hipStream_t st) {
    constexpr int block = norm_block(TPR), rpb = block / TPR;
    hipLaunchKernelGGL((rmsnorm_kernel<T, BITS, TPR, CPT>), flat_grid((a.n + rpb - 1) / rpb, block), dim3(block), 0, st,
                       (const T *)a.x, (const T *)a.residual, (const T *)a.weight, a.n, (int)a.d, 1.0 / a.d, a.eps,
                       (T *)a.h, (T *)a.y, (uint8_t *)a.y, (uint8_t *)a.scales, a.rstd);
    return hipGetLastError();
}

// Enough threads that no one holds more than 32 coordinates of a row.
template <typename T, int BITS>
hipError_t norm_dispatch(const NormArgs &a, hipStream_t st) {
    const int64_t chunks = BITS ? mx_padded(a.d) / 8 : (a.d + 7) / 8;
    if (chunks <= 16) return norm_launch<T, BITS, 16, 1>(a, st);
    if (chunks <= 32) return norm_launch<T, BITS, 16, 2>(a, st);
    if (chunks <= 64) return norm_launch<T, BITS, 64, 1>(a, st);
    if (chunks <= 128) return norm_launch<T, BITS, 64, 2>(a, st);
    if (chunks <= 192) return norm_launch<T, BITS, 64, 3>(a, st);
    if (chunks <= 256) return norm_launch<T, BITS, 64, 4>(a, st);
    if (chunks <= 512) return norm_launch<T, BITS, 256, 2>(a, st);
    if (chunks <= 1024) return norm_launch<T, BITS, 256, 4>(a, st);
    return norm_launch<T, BITS, 1024, 0>(a, st);
}

template <typename T>
hipError_t norm_typed(int format, const NormArgs &a, hipStream_t st) {
    if (format == MX_FP4) return norm_dispatch<T, 4>(a, st);
    if (format == MX_FP8) return norm_dispatch<T, 8>(a, st);
    return norm_dispatch<T, 0>(a, st);
}

template <typename T, int TPR, int CPT>
hipError_t grad_launch(const NormGradArgs &a, hipStream_t st) {
    hipLaunchKernelGGL((rmsnorm_grad_kernel<T, TPR, CPT>), dim3((unsigned)a.parts), dim3(256), 0, st, (const T *)a.dy,
                       (const T *)a.h, (const T *)a.weight, a.rstd, (const T *)a.dh, a.n, (int)a.d, (T *)a.dx,
                       a.dw ? a.partial : nullptr);
    return hipGetLastError();
}

template <typename T>
hipError_t grad_typed(const NormGradArgs &a, hipStream_t st) {
    const int64_t chunks = (a.d + 7) / 8;
    hipError_t e;
    if (chunks <= 16)
        e = grad_launch<T, 16, 1>(a, st);
    else if (chunks <= 32)
        e = grad_launch<T, 16, 2>(a, st);
    else if (chunks <= 64)
        e = grad_launch<T, 64, 1>(a, st);
    else if (chunks <= 128)
        e = grad_launch<T, 64, 2>(a, st);
    else if (chunks <= 192)
        e = grad_launch<T, 64, 3>(a, st);
    else if (chunks <= 256)
        e = grad_launch<T, 64, 4>(a, st);
    else if (chunks <= 512)
        e = grad_launch<T, 256, 2>(a, st);
    else if (chunks <= 1024)
        e = grad_launch<T, 256, 4>(a, st);
    else {
        // (a grid's x extent holds 2^22 rows of 1 024 threads)
        constexpr int64_t rows = int64_t(1) << 21;
        for (int64_t r = 0; r < a.n; r += rows)
            hipLaunchKernelGGL((rmsnorm_grad_long_kernel<T>), dim3((unsigned)std::min(rows, a.n - r)), dim3(1024), 0, st,
                               (const T *)a.dy + r * a.d, (const T *)a.h + r * a.d, (const T *)a.weight, a.rstd + r,
                               a.dh ? (const T *)a.dh + r * a.d : nullptr, (int)a.d, (T *)a.dx + r * a.d);
        e = hipGetLastError();
        if (e == hipSuccess && a.dw) {
            const int64_t per = (a.n + a.parts - 1) / a.parts;
            hipLaunchKernelGGL((rmsnorm_dw_long_kernel<T>), dim3((unsigned)((a.d + 255) / 256), (unsigned)a.parts),
                               dim3(256), 0, st, (const T *)a.dy, (const T *)a.h, a.rstd, a.n, (int)a.d, per, a.partial);
            e = hipGetLastError();
        }
    }
    if (e != hipSuccess || !a.dw) return e;
    hipLaunchKernelGGL(column_sum_kernel, dim3((unsigned)((a.d + kDwCols - 1) / kDwCols)), dim3(kDwCols * kDwRows), 0, st,
                       a.partial, (int)a.parts, (int)a.d, a.dw);
    return hipGetLastError();
}

}  // namespace

hipError_t launch_mx_quantize(int prec, int bits, const void *x, int64_t n, int64_t d, void *codes, void *scales,
                              hipStream_t st) {
    if (n == 0) return hipSuccess;
    if (prec == P_FP32) return bits == 4 ? quantize<float, 4>(x, n, d, codes, scales, st) : quantize<float, 8>(x, n, d, codes, scales, st);
    if (prec == P_FP16)
        return bits == 4 ? quantize<_Float16, 4>(x, n, d, codes, scales, st) : quantize<_Float16, 8>(x, n, d, codes, scales, st);
    return bits == 4 ? quantize<__bf16, 4>(x, n, d, codes, scales, st) : quantize<__bf16, 8>(x, n, d, codes, scales, st);
}

hipError_t launch_mx_dequantize(int prec, int bits, const void *codes, const void *scales, int64_t n, int64_t d, void *x,
                                hipStream_t st) {
    if (n == 0) return hipSuccess;
    if (prec == P_FP32)
        return bits == 4 ? dequantize<float, 4>(codes, scales, n, d, x, st) : dequantize<float, 8>(codes, scales, n, d, x, st);
    if (prec == P_FP16)
        return bits == 4 ? dequantize<_Float16, 4>(codes, scales, n, d, x, st)
                         : dequantize<_Float16, 8>(codes, scales, n, d, x, st);
    return bits == 4 ? dequantize<__bf16, 4>(codes, scales, n, d, x, st) : dequantize<__bf16, 8>(codes, scales, n, d, x, st);
}

hipError_t launch_rmsnorm(int prec, int format, const NormArgs &a, hipStream_t st) {
    if (a.n == 0) return hipSuccess;
    if (prec == P_FP32) return norm_typed<float>(format, a, st);
    if (prec == P_FP16) return norm_typed<_Float16>(format, a, st);
    return norm_typed<__bf16>(format, a, st);
}

int64_t rmsnorm_grad_parts(int64_t n, int64_t d) {
    const int64_t chunks = (d + 7) / 8;
    if (chunks > 1024) return std::min<int64_t>(n, 64);
    const int64_t rpb = chunks <= 32 ? 16 : chunks <= 256 ? 4 : 1;
    return std::min<int64_t>((n + rpb - 1) / rpb, 512);  // as many as are resident
}

hipError_t launch_rmsnorm_grad(int prec, const NormGradArgs &a, hipStream_t st) {
    if (prec == P_FP32) return grad_typed<float>(a, st);
    if (prec == P_FP16) return grad_typed<_Float16>(a, st);
    return grad_typed<__bf16>(a, st);
}

}  // namespace exemcl
