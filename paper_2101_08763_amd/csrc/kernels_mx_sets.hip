// kernels_mx_sets.hip -- sets on 4-bit rows: the choice of a kernel, and the one
// for long rows.
#include "mx_sets.hpp"

namespace exemcl {

namespace {

// biases[i] = -||s||^2 / 2 of slot i's row, one wavefront each, in 64 bits (the
// squares of a block's elements add up to a whole number of quarters).
__global__ __launch_bounds__(256) void mx_bias_kernel(const uint8_t *__restrict__ codes,
                                                      const uint8_t *__restrict__ scales, int64_t n, int64_t d,
                                                      const int32_t *__restrict__ sets, int64_t slots,
                                                      float *__restrict__ biases) {
    const int64_t i = flat_block() * 4 + (threadIdx.x >> 6);
    const int lane = threadIdx.x & 63;
    if (i >= slots) return;
    const int64_t s = sets[i];
    if (s < 0 || s >= n) {
        if (lane == 0) biases[i] = -FLT_MAX;
        return;
    }
    double q = 0.0;
    const int chunks = (int)(mx_padded(d) / 8);
    for (int c = lane; c < chunks; c += 64) {
        float v[8], e = 0.0f;
        mx_decode8<4>(u32x2{*reinterpret_cast<const uint32_t *>(codes + s * mx_row_bytes(d, 4) + c * 4), 0}, v);
#pragma unroll
        for (int j = 0; j < 8; ++j) e = fmaf(v[j], v[j], e);
        const double f = mx_factor(scales[s * mx_row_scales(d) + c / 4]);
        q += (double)e * f * f;
    }
#pragma unroll
    for (int off = 32; off >= 1; off >>= 1) q += __shfl_xor(q, off);
    if (lane == 0) biases[i] = (float)(-0.5 * q);
}

// Rows too long for registers: 32 points x 16 sets per wavefront, operands
// from memory.
__global__ __launch_bounds__(256) void mx_sets_direct_kernel(const uint8_t *__restrict__ codes,
                                                             const uint8_t *__restrict__ scales, int64_t n, int64_t d,
                                                             const int32_t *__restrict__ sets, int64_t l, int64_t k,
                                                             const float *__restrict__ biases, int64_t parts,
                                                             int64_t groups, float *__restrict__ partials, int64_t lpad) {
    const int lane = threadIdx.x & 63, lr = lane & 15, g = lane >> 4;
    const int64_t unit = flat_block() * 4 + (threadIdx.x >> 6), part = unit / groups, grp = unit - part * groups;
    if (part >= parts) return;
    const int64_t rb = mx_row_bytes(d, 4), rs = mx_row_scales(d);
    const int ksteps = (int)(mx_padded(d) / kMxRow);
    const int64_t r0 = min(part * kMxSetRows + lr, n - 1), r1 = min(part * kMxSetRows + 16 + lr, n - 1);
    const int64_t j = grp * 16 + lr;
    f32x4 m0 = {0.0f, 0.0f, 0.0f, 0.0f}, m1 = m0;
    for (int64_t p = 0; p < k; ++p) {
        const int64_t slot = min(j, l - 1) * k + p, s = sets[slot];
        const int64_t col = s >= 0 && s < n ? s : 0;
        const float b0 = biases[slot];
        f32x4 a0 = {b0, b0, b0, b0}, a1 = a0;
        for (int ks = 0; ks < ksteps; ++ks) {
            const int64_t at = ks * 64 + g * 16, sat = ks * 4 + g;
            const i32x4 b = *reinterpret_cast<const i32x4 *>(codes + col * rb + at);
            const int sb = scales[col * rs + sat];
            a0 = mx_mma(*reinterpret_cast<const i32x4 *>(codes + r0 * rb + at), b, a0, scales[r0 * rs + sat], sb);
            a1 = mx_mma(*reinterpret_cast<const i32x4 *>(codes + r1 * rb + at), b, a1, scales[r1 * rs + sat], sb);
        }
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            m0[i] = fmaxf(m0[i], a0[i]);
            m1[i] = fmaxf(m1[i], a1[i]);
        }
    }
    float t = 0.0f;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        if (part * kMxSetRows + 4 * g + i < n) t += m0[i];
        if (part * kMxSetRows + 16 + 4 * g + i < n) t += m1[i];
    }
    t += __shfl_xor(t, 16);
    t += __shfl_xor(t, 32);
    if (g == 0) partials[part * lpad + j] = t;
}

// Sums of kFold rows of partials, a thread per column and sum: the last pass has
// one workgroup per 16 sets, too few to read many rows at once.  Set scores of 16
// sets on 200 000, 1 000 000 points 18.7, 27.2 us (without 22.0, 71.9); from
// 100 000 points on (3 125 rows) it is worth its launch.
constexpr int kFold = 32;
constexpr int64_t kFoldFrom = 4096;

__global__ __launch_bounds__(256) void mx_fold_kernel(const float *__restrict__ partials, int64_t G, int64_t lpad,
                                                      int64_t l, float *__restrict__ folded) {
    const int64_t unit = flat_block() * 4 + (threadIdx.x >> 6), cols = (l + 63) / 64, f = unit / cols, g0 = f * kFold;
    const int64_t j = (unit - f * cols) * 64 + (threadIdx.x & 63);
    if (g0 >= G || j >= l) return;
    float x[kFold];
#pragma unroll
    for (int u = 0; u < kFold; ++u) x[u] = partials[min(g0 + u, G - 1) * lpad + j];
    double s = 0.0;
#pragma unroll
    for (int u = 0; u < kFold; ++u) s += g0 + u < G ? (double)x[u] : 0.0;
    folded[f * lpad + j] = (float)s;
}

hipError_t run_long(const MxSetsArgs &x, hipStream_t st) {
    const int64_t slots = x.l * x.k, groups = x.lpad / 16, parts = mx_sets_parts(x.n);
    hipLaunchKernelGGL(mx_bias_kernel, flat_grid((slots + 3) / 4, 256), dim3(256), 0, st, x.codes, x.scales, x.n, x.d, x.sets,
                       slots, (float *)x.work);
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
    hipLaunchKernelGGL(mx_sets_direct_kernel, flat_grid((parts * groups + 3) / 4, 256), dim3(256), 0, st, x.codes, x.scales,
                       x.n, x.d, x.sets, x.l, x.k, (const float *)x.work, parts, groups, x.partials, x.lpad);
    return hipGetLastError();
}

// Fragments per row: the next of the compiled numbers.
int mx_sets_bucket(int64_t d) {
    const int ksteps = (int)(mx_padded(d) / kMxRow);
    return ksteps <= 6 ? ksteps : (ksteps + 1) / 2 * 2;
}

}  // namespace

int64_t mx_sets_parts(int64_t n) { return (n + kMxSetRows - 1) / kMxSetRows; }

int64_t mx_sets_folds(int64_t G) { return G >= kFoldFrom ? (G + kFold - 1) / kFold : 0; }

hipError_t launch_mx_fold(const float *partials, int64_t G, int64_t lpad, int64_t l, float *folded, hipStream_t st) {
    const int64_t units = (G + kFold - 1) / kFold * ((l + 63) / 64);
    hipLaunchKernelGGL(mx_fold_kernel, flat_grid((units + 3) / 4, 256), dim3(256), 0, st, partials, G, lpad, l, folded);
    return hipGetLastError();
}

int64_t mx_sets_work(int64_t d, int64_t k) {
    if (d > kMxSetsD) return kMxSets * k * 4;
    const int ks = mx_sets_bucket(d);
    return (k + 1) / 2 * 2 * (ks * 1024 + (ks + 3) / 4 * 256 + 64);
}

hipError_t launch_mx_sets(const void *codes, const void *scales, int64_t n, int64_t d, const int32_t *sets, int64_t l,
                          int64_t k, void *work, float *partials, int64_t lpad, hipStream_t st) {
    const MxSetsArgs x{(const uint8_t *)codes, (const uint8_t *)scales, n, d, sets, l, k, (uint8_t *)work, partials, lpad};
    if (d > kMxSetsD) return run_long(x, st);
    const int ks = mx_sets_bucket(d);
    return ks <= 6 ? mx_sets_short(ks, x, st) : mx_sets_wide(ks, x, st);
}

}  // namespace exemcl
