// glu_rows.hpp -- the gated block and products of few rows, weights straight from
// memory to the matrix cores (instantiated in kernels_glu_rows.hip and
// kernels_w4_*.hip).
//
//   y[i][j] = sum_t x[i][t] W[j][t] + b[j],  or  a(g) u of two such sums.
//
// With few rows every weight is read once and used little, so what bounds this is
// the weights' bytes.  A wavefront takes tiles of 16 weights' rows as the first
// operand of 16x16x32 instructions and up to 16 MT rows of x as the second; both
// come from memory in operand order, without LDS.  The wavefronts of a workgroup
// take blocks of 128 coordinates in turn, and their sums are added in order
// through LDS at the end.  No temporary memory, and no order that a launch
// changes.  One row by two bf16 weights of 8 192 x 4 096 that no cache holds takes 27.4
// us (4.9 TB/s, a large copy's rate), one by 4 bits of 4 096 x 131 072 57 (5 TB/s), of
// 4 096 x 32 768 18 (4 TB/s); below 30 MB the launch and the first loads are most of it
// (7.0 us for 4 096 x 8 192 by 4 bits, 3.1 at the copy's rate).  16 wavefronts to a workgroup
// spill, and so does the block by 4 bits in groups of 32 with two tiles (w4_rows.hpp).
//
// Weights of 4 bits are whole numbers q = 0 .. 15 beside a scale s and a zero
// point z per group: sum x w = s (sum x q - z sum x).  The byte 0x0q read as E4M3
// is q 2^-9 (its subnormal and first binade are one line), so one conversion makes
// two operands of fp16 or bf16 exactly.  The products run on q, whose sum is in
// fp32; sum x comes from an instruction on ones, shared by all tiles, and s and z
// are applied in fp32 once per group.  No weight is rounded.
#pragma once

#include <algorithm>

#include "glu_device.hpp"
#include "mfma_kernels.hpp"
#include "w4_layout.hpp"

namespace exemcl {

constexpr int kRowsWaves = 8;


// Eight elements of a row of x or of 16- or 32-bit weights as operands.
template <typename T>
struct RowsFrag {
    using E = typename Operand<T>::E;
    using vec = typename Mfma<E, 16>::vec_t;
    vec part[Operand<T>::PARTS];
};

template <typename T>
__device__ __forceinline__ RowsFrag<T> rows_frag(typename Chunk<T>::vec v) {
    RowsFrag<T> r;
    if constexpr (sizeof(T) == 4) {
        f32x8 f;
#pragma unroll
        for (int e = 0; e < 8; ++e) f[e] = v[e];
        split_parts(f, r.part[0], r.part[1], r.part[2]);
    } else {
#pragma unroll
        for (int e = 0; e < 8; ++e) r.part[0][e] = v[e];
    }
    return r;
}

// acc + w x, both of type T.
template <typename T>
__device__ __forceinline__ f32x4 rows_mma(const RowsFrag<T> &w, const RowsFrag<T> &x, f32x4 acc) {
    using M = Mfma<typename Operand<T>::E, 16>;
#pragma unroll
    for (int p = Operand<T>::PRODUCTS - 1; p >= 0; --p) acc = M::mma(w.part[part_a(p)], x.part[part_b(p)], 0, acc);
    return acc;
}

// acc + w x for w exact in 16 bits.
template <typename T>
__device__ __forceinline__ f32x4 rows_mma_whole(typename RowsFrag<T>::vec w, const RowsFrag<T> &x, f32x4 acc) {
    using M = Mfma<typename Operand<T>::E, 16>;
#pragma unroll
    for (int p = Operand<T>::PARTS - 1; p >= 0; --p) acc = M::mma(w, x.part[p], 0, acc);
    return acc;
}

// The eight 4-bit numbers of a dword (exemcl.h has their order).
__device__ __forceinline__ bf16x8 w4_operand(uint32_t c, __bf16) {
    typedef __bf16 pair __attribute__((ext_vector_type(2)));
    const uint32_t lo = c & 0x0f0f0f0fu, hi = c >> 4 & 0x0f0f0f0fu;
    const pair a = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(lo, 512.0f, false), b = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(lo, 512.0f, true);
    const pair e = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(hi, 512.0f, false), g = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(hi, 512.0f, true);
    return bf16x8{a[0], a[1], b[0], b[1], e[0], e[1], g[0], g[1]};
}
__device__ __forceinline__ f16x8 w4_operand(uint32_t c, _Float16) {
    typedef _Float16 pair __attribute__((ext_vector_type(2)));
    const uint32_t lo = c & 0x0f0f0f0fu, hi = c >> 4 & 0x0f0f0f0fu;
    const pair a = __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(lo, 512.0f, false), b = __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(lo, 512.0f, true);
    const pair e = __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(hi, 512.0f, false), g = __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(hi, 512.0f, true);
    return f16x8{a[0], a[1], b[0], b[1], e[0], e[1], g[0], g[1]};
}

struct RowsArgs {
    const void *x;
    int64_t n, d;
    const void *w[2], *words[2];  // gate and up, or one
    int64_t f;
    const float *b[2];
    int act;
    void *y, *g, *u;
    uint32_t mblocks, units;
};

// GROUP 0: weights of type T; else 4-bit ones with so many to a group.  RT tiles
// of 16 weights' rows a wavefront (GLU: of both matrices), 16 MT rows of x; AHEAD
// blocks of a wavefront are loaded before the first is used.
template <typename T, int GROUP, bool GLU, int RT, int MT, int AHEAD>
__global__ __launch_bounds__(kRowsWaves * 64) void rows_kernel(const RowsArgs a) {
    using E = typename Operand<T>::E;
    using vec = typename Mfma<E, 16>::vec_t;
    constexpr int MATS = GLU ? 2 : 1, TILES = RT * MATS;
    constexpr int UNITS = RT * MT, MOST = 4 / MATS, PASS = UNITS < MOST ? UNITS : MOST;
    __shared__ f32x4 sums[kRowsWaves][PASS * MATS][64];
    const int lane = threadIdx.x & 63, lr = lane & 15, g = lane >> 4;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);

    // Workgroups b, b + 8, ... share an XCD: blocks of rows that read the same
    // weights follow each other there.
    const uint32_t wg = (uint32_t)flat_block(), pos = wg >> 3;
    const uint32_t turn = __builtin_amdgcn_readfirstlane(a.mblocks == 1 ? pos : pos / a.mblocks), unit = turn * 8 + (wg & 7);
    if (unit >= a.units) return;
    const int64_t tile0 = (int64_t)unit * RT, row0 = (int64_t)(pos - turn * a.mblocks) * (16 * MT);
    const int64_t d = a.d, ftiles = (a.f + 15) / 16;

    const T *x[MT];
#pragma unroll
    for (int m = 0; m < MT; ++m) x[m] = (const T *)a.x + min(row0 + m * 16 + lr, a.n - 1) * d;
    // The tiles' rows, past the last one it again.
    const T *w[TILES];
    const u32x4 *codes[TILES];
    const u32x4 *words[TILES];
#pragma unroll
    for (int t = 0; t < TILES; ++t) {
        const int64_t tile = min(tile0 + t / MATS, ftiles - 1);
        if constexpr (GROUP == 0) {
            w[t] = (const T *)a.w[t % MATS] + min(tile * 16 + lr, a.f - 1) * d;
        } else {
            codes[t] = (const u32x4 *)a.w[t % MATS] + tile * w4_blocks(d) * 64 + lane;
            words[t] = (const u32x4 *)a.words[t % MATS] + tile * w4_groups(d, GROUP) * 4 + g;
        }
    }

    f32x4 acc[TILES][MT];
#pragma unroll
    for (int t = 0; t < TILES; ++t)
#pragma unroll
        for (int m = 0; m < MT; ++m) acc[t][m] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};

    // Whole blocks; weights of type T in steps of 32 coordinates where these are fewer
    // than the wavefronts.
    const int blocks = (int)w4_blocks(d), full_blocks = (int)(d / kW4Block);
    const int whole = GROUP == 0 && full_blocks < kRowsWaves ? 0 : full_blocks;
    // A block as it comes from memory: the weights and their words, and x (many rows
    // of which are read when they are needed).
    constexpr bool HOLD = MT == 1;
    constexpr int STEPS = GROUP ? GROUP / 32 : 4, GPB = 4 / STEPS;  // instructions per group, groups per block
    struct Block {
        u32x4 c[GROUP ? TILES : 1], sz[GROUP ? TILES : 1][GPB];
        typename Chunk<T>::vec w[GROUP ? 1 : TILES][4], x[4];
    };
    auto chunk = [&](const T *row, int b, int j, auto full) {
        const int k = b * kW4Block + 32 * j + 8 * g;
        return load8(row + (full ? k : min((int64_t)k, d - 1)), full ? 8 : (int)(d - k));
    };
    auto load = [&](Block &r, int b, auto full) {
        if constexpr (GROUP == 0) {
#pragma unroll
            for (int t = 0; t < TILES; ++t)
#pragma unroll
                for (int j = 0; j < 4; ++j) r.w[t][j] = chunk(w[t], b, j, full);
        } else {
#pragma unroll
            for (int t = 0; t < TILES; ++t) {
                r.c[t] = codes[t][b * 64];
#pragma unroll
                for (int q = 0; q < GPB; ++q) r.sz[t][q] = words[t][(b * GPB + q) * 4];
            }
        }
        if constexpr (HOLD)
#pragma unroll
            for (int j = 0; j < 4; ++j) r.x[j] = chunk(x[0], b, j, full);
    };
    // 32 coordinates of weights of type T.
    auto step = [&](auto weights, auto rows) {
        RowsFrag<T> wf[TILES];
#pragma unroll
        for (int t = 0; t < TILES; ++t) wf[t] = weights(t);
#pragma unroll
        for (int m = 0; m < MT; ++m) {
            const RowsFrag<T> xf = rows(m);
#pragma unroll
            for (int t = 0; t < TILES; ++t) acc[t][m] = rows_mma<T>(wf[t], xf, acc[t][m]);
        }
    };
    auto use = [&](const Block &r, int b, auto full) {
        auto x_frag = [&](int m, int j) { return rows_frag<T>(HOLD ? r.x[j] : chunk(x[m], b, j, full)); };
        if constexpr (GROUP == 0) {
#pragma unroll
            for (int j = 0; j < 4; ++j)
                step([&](int t) { return rows_frag<T>(r.w[t][j]); }, [&](int m) { return x_frag(m, j); });
        } else {
            vec ones;
#pragma unroll
            for (int e = 0; e < 8; ++e) ones[e] = (E)1.0f;
#pragma unroll
            for (int q = 0; q < GPB; ++q) {
                RowsFrag<T> xf[MT][STEPS];
                float xs[MT];
#pragma unroll
                for (int m = 0; m < MT; ++m) {
                    f32x4 s = {0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
                    for (int j = 0; j < STEPS; ++j) {
                        xf[m][j] = x_frag(m, q * STEPS + j);
                        s = rows_mma_whole<T>(ones, xf[m][j], s);
                    }
                    xs[m] = s[0];
                }
#pragma unroll
                for (int t = 0; t < TILES; ++t) {
                    vec wf[STEPS];
#pragma unroll
                    for (int j = 0; j < STEPS; ++j) wf[j] = w4_operand(r.c[t][q * STEPS + j], E());
#pragma unroll
                    for (int m = 0; m < MT; ++m) {
                        f32x4 p = {0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
                        for (int j = 0; j < STEPS; ++j) p = rows_mma_whole<T>(wf[j], xf[m][j], p);
#pragma unroll
                        for (int i = 0; i < 4; ++i) {
                            const uint32_t word = r.sz[t][q][i];
                            acc[t][m][i] = fmaf(__uint_as_float(word & 0xffffff00u),
                                                fmaf(-(float)(word & 0xffu), xs[m], p[i]), acc[t][m][i]);
                        }
                    }
                }
            }
        }
    };
    for (int b0 = wave; b0 < whole; b0 += kRowsWaves * AHEAD) {
        Block r[AHEAD];
#pragma unroll
        for (int i = 0; i < AHEAD; ++i) load(r[i], min(b0 + i * kRowsWaves, whole - 1), std::true_type());
#pragma unroll
        for (int i = 0; i < AHEAD; ++i) {
            __builtin_amdgcn_sched_barrier(0);
            if (i == 0 || b0 + i * kRowsWaves < whole) use(r[i], b0 + i * kRowsWaves, std::true_type());
        }
    }
    if constexpr (GROUP == 0) {
#pragma unroll 1
        for (int j = wave; whole * kW4Block + 32 * j < d; j += kRowsWaves) {
            auto part = [&](const T *row) { return rows_frag<T>(chunk(row, whole, j, std::false_type())); };
            step([&](int t) { return part(w[t]); }, [&](int m) { return part(x[m]); });
        }
    } else if (whole < blocks && whole % kRowsWaves == wave) {
        Block r;
        load(r, whole, std::false_type());
        use(r, whole, std::false_type());
    }

    // The wavefronts' sums, PASS units of a tile and 16 rows at a time, each added
    // and finished by one wavefront.
#pragma unroll
    for (int u0 = 0; u0 < UNITS; u0 += PASS) {
        if (u0) __syncthreads();
#pragma unroll
        for (int i = 0; i < PASS; ++i)
            if (u0 + i < UNITS)
#pragma unroll
                for (int q = 0; q < MATS; ++q)
                    sums[wave][i * MATS + q][lane] = acc[(u0 + i) / MT * MATS + q][(u0 + i) % MT];
        __syncthreads();
        const int at = u0 + wave;
        if (wave < PASS && at < UNITS) {
            const int64_t row = row0 + at % MT * 16 + lr, col = (tile0 + at / MT) * 16 + 4 * g;
            const int have = (int)max((int64_t)0, min((int64_t)4, a.f - col));
            if (row < a.n && have > 0) {
                float v[MATS][4];
#pragma unroll
                for (int q = 0; q < MATS; ++q) {
                    f32x4 s = sums[0][wave * MATS + q][lane];
#pragma unroll
                    for (int w8 = 1; w8 < kRowsWaves; ++w8) s += sums[w8][wave * MATS + q][lane];
#pragma unroll
                    for (int i = 0; i < 4; ++i) v[q][i] = s[i] + (a.b[q] && i < have ? a.b[q][col + i] : 0.0f);
                }
                const int64_t to = row * a.f + col;
                if constexpr (GLU) {
                    if (a.g) store4((T *)a.g + to, have, v[0]);
                    if (a.u) store4((T *)a.u + to, have, v[1]);
                    with_activation(a.act, [&](auto act) {
#pragma unroll
                        for (int i = 0; i < 4; ++i)
                            v[0][i] = activation<decltype(act)::value, sizeof(T) == 2>(v[0][i]) * v[1][i];
                    });
                }
                store4((T *)a.y + to, have, v[0]);
            }
        }
    }
}

// Blocks of `rows` rows by units of `weights` weights' rows, 8 units at a time over
// the XCDs.
inline hipError_t rows_grid(RowsArgs &a, int64_t rows, int64_t weights) {
    const int64_t mblocks = (a.n + rows - 1) / rows, units = (a.f + weights - 1) / weights;
    if ((units + 7) / 8 > (int64_t(1) << 28) / mblocks) return hipErrorInvalidValue;  // 32 bits of workgroups
    a.mblocks = (uint32_t)mblocks, a.units = (uint32_t)units;
    return hipSuccess;
}
inline int64_t rows_workgroups(const RowsArgs &a) { return (int64_t)((a.units + 7) / 8) * 8 * a.mblocks; }

template <typename T, int GROUP, bool GLU, int RT, int MT, int AHEAD>
hipError_t rows_launch(RowsArgs a, hipStream_t st) {
    const hipError_t e = rows_grid(a, 16 * MT, 16 * RT);
    if (e != hipSuccess) return e;
    hipLaunchKernelGGL((rows_kernel<T, GROUP, GLU, RT, MT, AHEAD>), flat_grid(rows_workgroups(a), kRowsWaves * 64),
                       dim3(kRowsWaves * 64), 0, st, a);
    return hipGetLastError();
}

}  // namespace exemcl
