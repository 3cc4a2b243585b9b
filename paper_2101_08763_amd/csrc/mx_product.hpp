// mx_product.hpp -- products of microscaled rows, A (8 or 4 bits) with B (4
// bits): C[i][j] = sum_t A[i][t] B[j][t] + bias[j] (instantiated in
// kernels_mx_product_*.hip, one per format of A).
#pragma once

#include <algorithm>
#include <atomic>

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

// ---------------------------------------------------------------------------
// Tiles of C through LDS.  PM x PN wavefronts compute (16 WM PM) x (64 PN)
// elements, one K-step of 128 coordinates a stage, three stages in flight.  B's
// rows are the instruction's first operand, so a lane's accumulators lie along
// a row of C; fragment j of a wavefront holds B's rows 4 i + j (i = 0 .. 15) of
// its 64, which makes them 16 neighbours: a wavefront stores whole 128-byte
// lines of 16-bit results.  A's rows are dealt out the same way (row WM i + w in
// fragment w), so one LDS read gives a lane the scales of four fragments.
// ---------------------------------------------------------------------------
template <int BITS_A, int WM, int PM, int PN>
struct MxTilePlan {
    static constexpr int WAVES = PM * PN, THREADS = WAVES * 64, BM = PM * WM * 16, BN = PN * 64;
    static constexpr int A_FRAGS = PM * WM * BITS_A / 4, FRAGS = A_FRAGS + PN * 4;  // of 1 KiB
    static constexpr int SCALE_LOADS = (BM + BN) / 64;                              // of 64 rows
    static constexpr int LOADS = FRAGS / WAVES + SCALE_LOADS / WAVES;               // per thread and stage
    static constexpr int B_AT = A_FRAGS * 1024, AS_AT = FRAGS * 1024, BS_AT = AS_AT + BM * 4, BUF = BS_AT + BN * 4;
    static constexpr int LDS = 3 * BUF;
    static_assert(FRAGS % WAVES == 0 && SCALE_LOADS % WAVES == 0 && WM % 4 == 0 && LDS <= kLdsBytes, "geometry");
};

template <typename T, int BITS_A, bool DIVIDE, int WM, int PM, int PN>
__global__ __launch_bounds__(PM *PN * 64, 2) void mx_product_kernel(const uint8_t *__restrict__ A,
                                                                    const uint8_t *__restrict__ As, int64_t m,
                                                                    const uint8_t *__restrict__ B,
                                                                    const uint8_t *__restrict__ Bs, int64_t n, int ksteps,
                                                                    int mblocks, int nblocks,
                                                                    const float *__restrict__ bias, T *__restrict__ C) {
    using P = MxTilePlan<BITS_A, WM, PM, PN>;
    extern __shared__ __align__(16) unsigned char smem[];
    const int tid = threadIdx.x, lane = tid & 63, lr = lane & 15, g = lane >> 4;
    const int wave = __builtin_amdgcn_readfirstlane(tid >> 6), wm = wave % PM, wn = wave / PM;

    // Workgroups b, b + 8, b + 16, ... share an XCD and its L2: they take
    // consecutive tiles, up to 8 of one row of tiles side by side.
    const int64_t units = (int64_t)mblocks * nblocks, per = (units + 7) / 8;
    const int64_t b = flat_block(), pos = b >> 3, u = (b & 7) * per + pos;
    if (pos >= per || u >= units) return;
    const int64_t strip = u / ((int64_t)mblocks * 8);
    const int width = (int)min((int64_t)8, nblocks - strip * 8);
    const int64_t in = u - strip * mblocks * 8;
    const int64_t m0 = in / width * P::BM, n0 = (strip * 8 + in % width) * P::BN;

    const int a_row = ksteps * 16 * BITS_A, b_row = ksteps * 64, s_row = ksteps * 4;
    const uint32_t mrows = (uint32_t)min((int64_t)P::BM, m - m0), nrows = (uint32_t)min((int64_t)P::BN, n - n0);
    const auto awin = window_rsrc(A + m0 * a_row, mrows * (uint32_t)a_row);
    const auto bwin = window_rsrc(B + n0 * b_row, nrows * (uint32_t)b_row);
    const auto aswin = window_rsrc(As + m0 * s_row, mrows * (uint32_t)s_row);
    const auto bswin = window_rsrc(Bs + n0 * s_row, nrows * (uint32_t)s_row);

    // What lies past the rows, or in stages past the last, reads as zeros.
    auto issue = [&](int st) {
        unsigned char *buf = smem + st % 3 * P::BUF;
        const bool live = st < ksteps;
#pragma unroll
        for (int i = 0; i < P::FRAGS / P::WAVES; ++i) {
            const int f = i * P::WAVES + wave;
            if (f < P::A_FRAGS) {
                constexpr int H = BITS_A / 4;  // halves of a fragment
                const int w = f / H % WM, block = f / H / WM;
                const int row = block * WM * 16 + lr * WM + w;
                const uint32_t off = (uint32_t)row * a_row + st * (16 * BITS_A) + f % H * 64 + g * 16;
                window_to_lds16(awin, buf + f * 1024, live ? off : kDeadOffset);
            } else {
                const int j = (f - P::A_FRAGS) % 4, block = (f - P::A_FRAGS) / 4;
                const int row = block * 64 + lr * 4 + j;
                window_to_lds16(bwin, buf + f * 1024, live ? (uint32_t)row * b_row + st * 64 + g * 16 : kDeadOffset);
            }
        }
#pragma unroll
        for (int i = 0; i < P::SCALE_LOADS / P::WAVES; ++i) {
            const int f = i * P::WAVES + wave;
            const int row = (f * 64 < P::BM ? f * 64 : f * 64 - P::BM) + lane;
            const uint32_t off = live ? (uint32_t)row * s_row + st * 4 : kDeadOffset;
            if (f * 64 < P::BM)
                window_to_lds4(aswin, buf + P::AS_AT + f * 256, off);
            else
                window_to_lds4(bswin, buf + P::AS_AT + f * 256, off);
        }
    };

    f32x4 acc[WM][4];
#pragma unroll
    for (int w = 0; w < WM; ++w)
#pragma unroll
        for (int j = 0; j < 4; ++j) acc[w][j] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};

    issue(0);
    issue(1);
    for (int st = 0; st < ksteps; ++st) {
        asm volatile("s_waitcnt vmcnt(%0)" ::"n"(P::LOADS) : "memory");
        __syncthreads();
        issue(st + 2);
        const unsigned char *buf = smem + st % 3 * P::BUF;
        const i32x4 *af = reinterpret_cast<const i32x4 *>(buf) + wm * WM * (BITS_A / 4) * 64 + lane;
        const i32x4 *bf = reinterpret_cast<const i32x4 *>(buf + P::B_AT) + wn * 4 * 64 + lane;
        i32x4 bx[4];
#pragma unroll
        for (int j = 0; j < 4; ++j) bx[j] = bf[j * 64];
        i32x4 bs = *reinterpret_cast<const i32x4 *>(buf + P::BS_AT + (wn * 64 + lr * 4) * 4);
#pragma unroll
        for (int j = 0; j < 4; ++j) bs[j] = (int)((uint32_t)bs[j] >> (8 * g));  // the low byte counts
#pragma unroll
        for (int w0 = 0; w0 < WM; w0 += 4) {
            i32x4 as = *reinterpret_cast<const i32x4 *>(buf + P::AS_AT + (wm * WM * 16 + lr * WM + w0) * 4);
#pragma unroll
            for (int i = 0; i < 4; ++i) as[i] = (int)((uint32_t)as[i] >> (8 * g));
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const int w = w0 + i;
                if constexpr (BITS_A == 4) {
                    const i32x4 ax = af[w * 64];
#pragma unroll
                    for (int j = 0; j < 4; ++j) acc[w][j] = mx_mma(bx[j], ax, acc[w][j], bs[j], as[i]);
                } else {
                    const i32x8 ax = mx_join(af[w * 128], af[w * 128 + 64]);
                    if constexpr (DIVIDE) {
                        i32x8 high, low;
                        mx_divide(ax, high, low);
#pragma unroll
                        for (int j = 0; j < 4; ++j) acc[w][j] = mx_mma(bx[j], low, acc[w][j], bs[j], as[i]);
#pragma unroll
                        for (int j = 0; j < 4; ++j) acc[w][j] = mx_mma(bx[j], high, acc[w][j], bs[j], as[i]);
                    } else {
#pragma unroll
                        for (int j = 0; j < 4; ++j) acc[w][j] = mx_mma(bx[j], ax, acc[w][j], bs[j], as[i]);
                    }
                }
            }
        }
    }
    asm volatile("s_waitcnt vmcnt(0)" ::: "memory");  // the last copies

    // Accumulator i of fragment j is column 16 g + 4 i + j of the wavefront's 64.
    const int64_t col = n0 + wn * 64 + g * 16;
    const int have = (int)max((int64_t)0, min((int64_t)16, n - col));
    float bb[16];
#pragma unroll
    for (int e = 0; e < 16; ++e) bb[e] = bias && e < have ? bias[col + e] : 0.0f;
#pragma unroll
    for (int w = 0; w < WM; ++w) {
        const int64_t row = m0 + wm * WM * 16 + lr * WM + w;
        float lo[8], hi[8];
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            lo[e] = acc[w][e % 4][e / 4] + bb[e];
            hi[e] = acc[w][e % 4][e / 4 + 2] + bb[e + 8];
        }
        if (row < m) {
            T *c = C + row * n + col;
            store8(c, have, lo);
            store8(c + 8, have - 8, hi);
        }
    }
}

template <typename T, int BITS_A, bool DIVIDE>
hipError_t product_direct(const MxProductArgs &a, hipStream_t st) {
    const int64_t mt = (a.m + 15) / 16, nt = (a.n + 15) / 16;
    if (mt > (int64_t(1) << 34) / nt) return hipErrorInvalidValue;  // 2^14 rows of kFlatRow
    hipLaunchKernelGGL((mx_product_direct_kernel<T, BITS_A, DIVIDE>), flat_grid(mt * nt, kDirectWaves * 64),
                       dim3(kDirectWaves * 64), 0, st, (const uint8_t *)a.A, (const uint8_t *)a.A_scales, a.m,
                       (const uint8_t *)a.B, (const uint8_t *)a.B_scales, a.n, a.d, nt, a.bias, (T *)a.C);
    return hipGetLastError();
}

template <typename T, int BITS_A, bool DIVIDE, int WM, int PM, int PN>
hipError_t product_tiled(const MxProductArgs &a, hipStream_t st) {
    using P = MxTilePlan<BITS_A, WM, PM, PN>;
    auto kern = mx_product_kernel<T, BITS_A, DIVIDE, WM, PM, PN>;
    static std::atomic<bool> ready[kMaxDevices];  // the attribute holds for one device
    const int dev = current_device();
    if (dev < 0) return hipErrorInvalidDevice;
    if (!ready[dev].load(std::memory_order_acquire)) {
        const hipError_t e = hipFuncSetAttribute((const void *)kern, hipFuncAttributeMaxDynamicSharedMemorySize, P::LDS);
        if (e != hipSuccess) return e;
        ready[dev].store(true, std::memory_order_release);
    }
    const int64_t mb = (a.m + P::BM - 1) / P::BM, nb = (a.n + P::BN - 1) / P::BN;
    if (mb > (int64_t(1) << 34) / nb) return hipErrorInvalidValue;
    hipLaunchKernelGGL(kern, flat_grid((mb * nb + 7) / 8 * 8, P::THREADS), dim3(P::THREADS), P::LDS, st,
                       (const uint8_t *)a.A, (const uint8_t *)a.A_scales, a.m, (const uint8_t *)a.B,
                       (const uint8_t *)a.B_scales, a.n, (int)(mx_padded(a.d) / kMxRow), (int)mb, (int)nb, a.bias, (T *)a.C);
    return hipGetLastError();
}

template <typename T, int BITS_A, bool DIVIDE>
hipError_t product_run(const MxProductArgs &a, hipStream_t st) {
    if (a.m <= 16) return product_direct<T, BITS_A, DIVIDE>(a, st);
    // Rounds of workgroups over the CUs (two small ones to each), times a
    // tile's area.
    const int64_t cus = std::max<int64_t>(1, device_cu_count());
    auto tiles = [&](int64_t bm, int64_t bn) { return ((a.m + bm - 1) / bm) * ((a.n + bn - 1) / bn); };
    const int64_t large = (tiles(256, 256) + cus - 1) / cus * 4, small = (tiles(128, 128) + 2 * cus - 1) / (2 * cus) * 2;
    return large <= small * 1.25 ? product_tiled<T, BITS_A, DIVIDE, 8, 2, 4>(a, st)
                                 : product_tiled<T, BITS_A, DIVIDE, 4, 2, 2>(a, st);
}

// DIVIDE: 8-bit rows in two parts (mx_divide), for results in fp32; what the
// matrix cores drop otherwise is far below the rounding of a 16-bit result.
template <int BITS_A>
hipError_t product_typed(int prec, const MxProductArgs &a, hipStream_t st) {
    if (prec == P_FP32) return product_run<float, BITS_A, BITS_A == 8>(a, st);
    if (prec == P_FP16) return product_run<_Float16, BITS_A, false>(a, st);
    return product_run<__bf16, BITS_A, false>(a, st);
}

}  // namespace exemcl
