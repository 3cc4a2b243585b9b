// kernels_glu_point.hip -- the gated block's element-wise part of the gradient, and
// rows laid out as operands of the tiled products.
#include <algorithm>
#include <type_traits>

#include "glu_device.hpp"
#include "glu_stage.hpp"
#include "mfma_kernels.hpp"

namespace exemcl {

namespace {

// Eight values as operands at p: themselves, or their three parts in planes.
template <typename T>
__device__ __forceinline__ void store_operand(typename Operand<T>::E *p, int64_t plane, const float (&v)[8]) {
    using E = typename Operand<T>::E;
    typedef E vec __attribute__((ext_vector_type(8)));
    if constexpr (sizeof(T) == 4) {
        f32x8 f;
#pragma unroll
        for (int i = 0; i < 8; ++i) f[i] = v[i];
        bf16x8 h, m, l;
        split_parts(f, h, m, l);
        *reinterpret_cast<vec *>(p) = h;
        *reinterpret_cast<vec *>(p + plane) = m;
        *reinterpret_cast<vec *>(p + 2 * plane) = l;
    } else {
        vec x;
#pragma unroll
        for (int i = 0; i < 8; ++i) x[i] = (E)v[i];
        *reinterpret_cast<vec *>(p) = x;
    }
}

// Rows as operands; T: float, or uint16_t for either 16-bit type.
template <typename T>
__device__ __forceinline__ void stage_rows(const StageJobs &jobs, int64_t b) {
    const StagePlace at = stage_place(jobs, b, threadIdx.x);
    if (at.job < 0) return;
    const DenseStageJob j = jobs.job[at.job];
    const T *src = (const T *)j.src + at.row * j.d + at.c;
    const int have = (int)min((int64_t)8, j.d - at.c);
    if constexpr (sizeof(T) == 4) {
        float v[8];
        load8(src, have, v);
        store_operand<T>((__bf16 *)j.dst + at.row * at.ld + at.c, j.n * at.ld, v);
    } else {
        typedef T vec __attribute__((ext_vector_type(8)));
        *reinterpret_cast<vec *>((T *)j.dst + at.row * at.ld + at.c) = load8(src, have);
    }
}
template <typename T>
__global__ __launch_bounds__(kStageThreads) void dense_stage_kernel(const StageJobs jobs) {
    stage_rows<T>(jobs, flat_block());
}

__global__ __launch_bounds__(256) void zero_bytes_kernel(uint16_t *__restrict__ p, int64_t count) {
    for (int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x; i < count; i += (int64_t)gridDim.x * 256) p[i] = 0;
}

// dg = dh u a'(g), du = dh a(g).  A thread takes 8 columns of the rows r, r + 8,
// ... of a part.  HBM-bound: three reads and two writes (16 384 x 8 192 of bf16 229 us,
// 5.9 TB/s; 8 192 x 4 096 55, 6.1).  Rows to lay out for the products ride along as
// further workgroups: a launch less, 6 us of 35 where n d f is small.
//
// dg and du are rounded to the type of the products' operands (fp32: three parts, all
// of it), as a gradient that is kept in that type would be: half a step, 2^-9 of bf16 and
// 2^-12 of fp16, beside the same of the results (off by 0.0023 of a bf16 gradient's norm,
// by 0.0017 without).  A second part of each would double the products' instructions,
// which are what bounds the call.  The column sums add dg and du as they are before that
// rounding, in fp32 within a part.
constexpr int kPointCols = 32, kPointRows = 8;
static_assert(kPointCols * kPointRows == kStageThreads, "both kinds of workgroups in one launch");
template <typename T, int ACT>
__global__ __launch_bounds__(kPointCols *kPointRows) void glu_point_kernel(
    const T *__restrict__ dh, const T *__restrict__ gate, const T *__restrict__ up, int64_t n, int64_t f, int64_t ld,
    int64_t rows, uint32_t cblocks, int64_t parts, typename Operand<T>::E *__restrict__ dg,
    typename Operand<T>::E *__restrict__ du, float *__restrict__ sums, const StageJobs jobs) {
    using Raw = typename std::conditional<sizeof(T) == 4, float, uint16_t>::type;
    const int64_t own = cblocks * parts, block = flat_block();
    if (block >= own) return stage_rows<Raw>(jobs, block - own);
    __shared__ float part[kPointRows][kPointCols][17];
    const int cl = threadIdx.x % kPointCols, r = threadIdx.x / kPointCols;
    const uint32_t p = (uint32_t)block / cblocks, cb = (uint32_t)block - p * cblocks;
    const int64_t c = ((int64_t)cb * kPointCols + cl) * 8, r0 = p * rows, r1 = min(n, r0 + rows);
    const int have = (int)max((int64_t)0, min((int64_t)8, f - c));
    float sg[8] = {}, su[8] = {};
    if (c < ld)
        for (int64_t row = r0 + r; row < r1; row += kPointRows) {
            float d[8], g[8], u[8], og[8], ou[8];
            load8<true>(dh + row * f + c, have, d);
            load8<true>(gate + row * f + c, have, g);
            load8<true>(up + row * f + c, have, u);
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                float slope;
                const float a = activation<ACT, sizeof(T) == 2, true>(g[i], slope);
                og[i] = d[i] * u[i] * slope;
                ou[i] = d[i] * a;
                sg[i] += og[i];
                su[i] += ou[i];
            }
            store_operand<T>(dg + row * ld + c, n * ld, og);
            store_operand<T>(du + row * ld + c, n * ld, ou);
        }
    if (!sums) return;
#pragma unroll
    for (int i = 0; i < 8; ++i) part[r][cl][i] = sg[i], part[r][cl][8 + i] = su[i];
    __syncthreads();
    if (r >= 2) return;  // one for dg's sums, one for du's
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        float s = 0.0f;
#pragma unroll
        for (int q = 0; q < kPointRows; ++q) s += part[q][cl][r * 8 + i];
        if (i < have) sums[(r * parts + p) * f + c + i] = s;
    }
}

template <typename T>
hipError_t point(const GluPointArgs &a, hipStream_t st) {
    using E = typename Operand<T>::E;
    const int64_t ld = dense_ld(a.f), cb = (ld / 8 + kPointCols - 1) / kPointCols;
    const int64_t rows = (a.n + a.parts - 1) / a.parts;
    StageJobs jobs{};
    const int64_t blocks = cb * a.parts + stage_jobs(a.jobs, a.job_count, &jobs);
    if (blocks > int64_t(1) << 34) return hipErrorInvalidValue;
    auto go = [&](auto kern) {
        hipLaunchKernelGGL(kern, flat_grid(blocks, 256), dim3(256), 0, st, (const T *)a.dh, (const T *)a.g, (const T *)a.u,
                           a.n, a.f, ld, rows, (uint32_t)cb, a.parts, (E *)a.dg, (E *)a.du, a.sums, jobs);
    };
    if (a.act == ACT_SILU)
        go(glu_point_kernel<T, ACT_SILU>);
    else if (a.act == ACT_GELU)
        go(glu_point_kernel<T, ACT_GELU>);
    else if (a.act == ACT_GELU_TANH)
        go(glu_point_kernel<T, ACT_GELU_TANH>);
    else
        go(glu_point_kernel<T, ACT_RELU>);
    return hipGetLastError();
}

template <typename T>
hipError_t stage(const DenseStageJob *jobs, int count, hipStream_t st) {
    StageJobs s{};
    const int64_t blocks = stage_jobs(jobs, count, &s);
    if (blocks > int64_t(1) << 34) return hipErrorInvalidValue;
    if (blocks == 0) return hipSuccess;
    hipLaunchKernelGGL(dense_stage_kernel<T>, flat_grid(blocks, kStageThreads), dim3(kStageThreads), 0, st, s);
    return hipGetLastError();
}

}  // namespace

int64_t dense_ld(int64_t d) { return (d + 7) / 8 * 8; }
int dense_planes(int prec) { return prec == P_FP32 ? 3 : 1; }
bool dense_in_place(int prec, const void *p, int64_t d) { return prec != P_FP32 && d % 8 == 0 && (uintptr_t)p % 16 == 0; }

hipError_t launch_dense_stage(int prec, const DenseStageJob *jobs, int count, hipStream_t st) {
    return prec == P_FP32 ? stage<float>(jobs, count, st) : stage<uint16_t>(jobs, count, st);
}

// Enough workgroups for the chip, of 64 rows and more where there are many (us with
// the column sums, mean of 8 192 x 4 096, 16 384 x 8 192 and 2 000 x 512 of bf16: 1 024
// workgroups 107, 2 048 110, 4 096 103, 16 384 104).
int64_t glu_point_parts(int64_t n, int64_t f) {
    const int64_t cb = (dense_ld(f) / 8 + kPointCols - 1) / kPointCols;
    const int64_t most = std::min<int64_t>((n + kPointRows - 1) / kPointRows, 512);
    const int64_t parts = std::max<int64_t>(1, std::min(most, (4096 + cb - 1) / cb)), rows = (n + parts - 1) / parts;
    return (n + rows - 1) / rows;
}

hipError_t launch_zero_bytes(void *p, int64_t bytes, hipStream_t st) {
    const int64_t count = bytes / 2, blocks = std::min<int64_t>((count + 255) / 256, 4096);
    if (count == 0) return hipSuccess;
    hipLaunchKernelGGL(zero_bytes_kernel, dim3((unsigned)blocks), dim3(256), 0, st, (uint16_t *)p, count);
    return hipGetLastError();
}

hipError_t launch_glu_point(int prec, const GluPointArgs &a, hipStream_t st) {
    if (prec == P_FP32) return point<float>(a, st);
    if (prec == P_FP16) return point<_Float16>(a, st);
    return point<__bf16>(a, st);
}

}  // namespace exemcl
