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

// Rows too long for registers: 64 points x 16 sets per wavefront, four members of
// each set at a time, operands from memory: eight loads to 16 instructions, and
// the loads, 16 rows at once, bound it (20 000 x 2 304, 512 sets of 16: 892 us,
// 0.85 PFLOP/s; 32 points and one member at a time 2 525).
constexpr int kLongTiles = 4, kLongMembers = 4;

__global__ __launch_bounds__(256, 2) void mx_sets_long_kernel(const uint8_t *__restrict__ codes,
                                                              const uint8_t *__restrict__ scales, int64_t n, int64_t d,
                                                              const int32_t *__restrict__ sets, int64_t l, int64_t k,
                                                              const float *__restrict__ biases, int64_t blocks,
                                                              int64_t groups, float *__restrict__ partials, int64_t lpad) {
    constexpr int RT = kLongTiles, MB = kLongMembers;
    const int lane = threadIdx.x & 63, lr = lane & 15, g = lane >> 4;
    const int64_t unit = flat_block() * 4 + (threadIdx.x >> 6), block = unit / groups, grp = unit - block * groups;
    if (block >= blocks) return;
    const int64_t rb = mx_row_bytes(d, 4), rs = mx_row_scales(d), row0 = block * RT * 16, j = grp * 16 + lr;
    const int ksteps = (int)(mx_padded(d) / kMxRow);
    const uint8_t *a_row[RT], *as_row[RT];
#pragma unroll
    for (int t = 0; t < RT; ++t) {
        const int64_t r = min(row0 + t * 16 + lr, n - 1);
        a_row[t] = codes + r * rb + g * 16;
        as_row[t] = scales + r * rs + g;
    }
    f32x4 m[RT];
#pragma unroll
    for (int t = 0; t < RT; ++t) m[t] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};  // e0
    for (int64_t p0 = 0; p0 < k; p0 += MB) {
        const uint8_t *b_row[MB], *bs_row[MB];
        f32x4 acc[RT][MB];
#pragma unroll
        for (int q = 0; q < MB; ++q) {
            const int64_t slot = min(j, l - 1) * k + min(p0 + q, k - 1), s = sets[slot];
            const int64_t col = s >= 0 && s < n ? s : 0;
            const float bias = biases[slot];
            b_row[q] = codes + col * rb + g * 16;
            bs_row[q] = scales + col * rs + g;
#pragma unroll
            for (int t = 0; t < RT; ++t) acc[t][q] = f32x4{bias, bias, bias, bias};
        }
        for (int ks = 0; ks < ksteps; ++ks) {
            i32x4 a[RT], b[MB];
            int sa[RT], sb[MB];
#pragma unroll
            for (int q = 0; q < MB; ++q) {
                b[q] = *reinterpret_cast<const i32x4 *>(b_row[q] + ks * 64);
                sb[q] = bs_row[q][ks * 4];
            }
#pragma unroll
            for (int t = 0; t < RT; ++t) {
                a[t] = *reinterpret_cast<const i32x4 *>(a_row[t] + ks * 64);
                sa[t] = as_row[t][ks * 4];
            }
#pragma unroll
            for (int t = 0; t < RT; ++t)
#pragma unroll
                for (int q = 0; q < MB; ++q) acc[t][q] = mx_mma(a[t], b[q], acc[t][q], sa[t], sb[q]);
        }
        // (past the last member, it once more)
#pragma unroll
        for (int t = 0; t < RT; ++t)
#pragma unroll
            for (int q = 0; q < MB; ++q)
#pragma unroll
                for (int i = 0; i < 4; ++i) m[t][i] = fmaxf(m[t][i], acc[t][q][i]);
    }
#pragma unroll
    for (int h = 0; h < RT / 2; ++h) {
        float s = 0.0f;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            if (row0 + h * 32 + 4 * g + i < n) s += m[2 * h][i];
            if (row0 + h * 32 + 16 + 4 * g + i < n) s += m[2 * h + 1][i];
        }
        s += __shfl_xor(s, 16);
        s += __shfl_xor(s, 32);
        const int64_t part = row0 / kMxSetRows + h;
        if (g == 0 && part * kMxSetRows < n) partials[part * lpad + j] = s;
    }
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
    const int64_t slots = x.l * x.k, groups = x.lpad / 16, blocks = (x.n + kLongTiles * 16 - 1) / (kLongTiles * 16);
    hipLaunchKernelGGL(mx_bias_kernel, flat_grid((slots + 3) / 4, 256), dim3(256), 0, st, x.codes, x.scales, x.n, x.d, x.sets,
                       slots, (float *)x.work);
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
    hipLaunchKernelGGL(mx_sets_long_kernel, flat_grid((blocks * groups + 3) / 4, 256), dim3(256), 0, st, x.codes, x.scales,
                       x.n, x.d, x.sets, x.l, x.k, (const float *)x.work, blocks, groups, x.partials, x.lpad);
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
