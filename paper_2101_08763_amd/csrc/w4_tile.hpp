// w4_tile.hpp -- products by 4-bit weights and the gated block on them for many
// rows (instantiated in kernels_w4_*.hip).
//
// The arithmetic is that of glu_rows.hpp: instructions on whole numbers q, the sum
// of a group's x beside them, scale and zero point applied in fp32 once per group.
// Here a workgroup of 8 wavefronts computes 128 rows of x (fp32: 64) by 256 weights'
// rows (GLU: 128 of each matrix), 128 coordinates a stage.  Wavefront w loads the 16 rows of x
// that are tile w, which is operand order: its registers go to LDS as they are
// (fp32: in parts, made once) and to one instruction on ones for the sums.  A
// wavefront has 4 x 4 tiles of results (fp32: 4 x 2); its weights come from memory, a
// stage ahead, and are converted once for its tiles of x.
//
// What bounds it is the VALU beside the matrix cores: for 16 instructions on a group
// of 128 a tile converts 32 pairs and applies scale and zero point with 16 FMAs.
// 2 048 x 4 096 x 8 192 of bf16 by groups of 128 take 142 us, 0.97 PFLOP/s, the matrix
// cores busy 46 % of the cycles; by 64 and 32 it takes 5 and 32 % more (twice and four
// times the scales and zero points), of fp32 2.2 times as long (three parts).  Leaving
// out the FMAs, or the staging of x, would save a fifth each.  The VALU is busy 53 %,
// and a wavefront waits for 29 % of its time: behind the barrier all read their next x
// together.  Registers for it twice, or a third wavefront to a SIMD, do not fit (256
// are in use).  VALU and matrix phases held apart by barriers took 9 % more, and a
// higher priority for half of the wavefronts or hints to the compiler's scheduling
// changed nothing.
#pragma once

#include <atomic>

#include "glu_rows.hpp"

namespace exemcl {

template <typename T, int GROUP>
struct W4TilePlan {
    static constexpr int WAVES = 8, THREADS = WAVES * 64, RT = 4, WN = 4, WM = 2;
    static constexpr int PARTS = Operand<T>::PARTS, MT = PARTS == 1 ? 4 : 2, XT = WM * MT, ROWS = XT * 16;
    static constexpr int GPB = kW4Block / GROUP, STEPS = GROUP / 32;  // groups of a block, instructions of a group
    static constexpr int UNITS = RT * GPB;                            // of a block: a tile, a group
    static constexpr int SPW = XT * 4 / WAVES;                        // steps of x that a wavefront loads
    static constexpr int SUMS = GPB > 4 / SPW ? GPB : 4 / SPW;        // partial sums of x in a block
    static constexpr int X = XT * 4 * PARTS * 1024;                   // bytes of a block's x
    static constexpr int XS = SUMS * ROWS * 4;                        // its sums
    static constexpr int S = WN * RT * GPB * 64;                      // scales; minus zero points
    static constexpr int XS_AT = 2 * X, S_AT = XS_AT + 4 * XS, Z_AT = S_AT + 4 * S, LDS = Z_AT + 4 * S;
    static_assert(LDS <= kLdsBytes, "geometry");
};

// f(0), f(1), ... f(N - 1), the numbers as constants.
template <int N, int I = 0, typename F>
__device__ __forceinline__ void each(F &&f) {
    if constexpr (I < N) {
        f(std::integral_constant<int, I>());
        each<N, I + 1>(f);
    }
}

template <typename T, int GROUP, bool GLU>
__global__ __launch_bounds__(512, 2) void w4_tile_kernel(const RowsArgs a) {
    using P = W4TilePlan<T, GROUP>;
    using E = typename Operand<T>::E;
    using vec = typename Mfma<E, 16>::vec_t;
    constexpr int RT = P::RT, MT = P::MT, GPB = P::GPB, STEPS = P::STEPS, PARTS = P::PARTS, MATS = GLU ? 2 : 1;
    constexpr int UNITS = P::UNITS, SPW = P::SPW, SUMS = P::SUMS;
    constexpr bool AHEAD = GROUP < 128;  // a second set of codes
    extern __shared__ __align__(16) unsigned char smem[];
    const int lane = threadIdx.x & 63, lr = lane & 15, g = lane >> 4;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), wm = wave & 1, wn = wave >> 1;

    // Workgroups b, b + 8, ... share an XCD and its L2: blocks of rows that read the
    // same weights follow each other there.
    const uint32_t wg = (uint32_t)flat_block(), pos = wg >> 3;
    const int turn = __builtin_amdgcn_readfirstlane(pos / a.mblocks), unit = turn * 8 + (int)(wg & 7);
    if ((uint32_t)unit >= a.units) return;
    const int d = (int)a.d, blocks = (int)w4_blocks(d), whole = d / kW4Block;
    const int64_t row0 = (int64_t)((int)pos - turn * (int)a.mblocks) * P::ROWS;
    const int tile0 = unit * (P::WN * RT / MATS), ftiles = (int)((a.f + 15) / 16);

    // Tile t of the workgroup's 16 (GLU: gate and up in turn), past the last one it
    // again.
    auto tile_of = [&](int t) { return (int64_t)min(tile0 + t / MATS, ftiles - 1); };
    const u32x4 *codes[RT];
#pragma unroll
    for (int t = 0; t < RT; ++t) codes[t] = (const u32x4 *)a.w[t % MATS] + tile_of(wn * RT + t) * blocks * 64;
    // This wavefront brings steps step0 .. of tile xt of x, in operand order, and the
    // words of two tiles: lane (lr, g) those of row lr for group g (past the last one
    // it again).
    const int xt = wave % P::XT, step0 = wave / P::XT * SPW, col0 = 32 * step0 + 8 * g;
    const int64_t xrow = min(row0 + xt * 16, a.n - 1);
    const T *x = (const T *)a.x + xrow * d;
    const int xrow_at = (int)min((int64_t)lr, a.n - 1 - xrow) * d;
    const int word_at = min(g, GPB - 1) * 16 + lr;
    const uint32_t *words[2];
#pragma unroll
    for (int i = 0; i < 2; ++i) {
        const int t = wave * 2 + i;
        words[i] = (const uint32_t *)a.words[t % MATS] + tile_of(t) * blocks * GPB * 16;
    }

    typename Chunk<T>::vec xr[SPW];
    uint32_t wr[2];
    u32x4 c[RT], cr[AHEAD ? RT : 1];
    // Past the last block it again, never used.
    auto load_codes = [&](int t, int b) { return (codes[t] + (int64_t)min(b, blocks - 1) * 64)[lane]; };
    auto load = [&](int b, auto full) {
        const int at = min(b, blocks - 1);
#pragma unroll
        for (int i = 0; i < 2; ++i) wr[i] = (words[i] + (int64_t)at * GPB * 16)[word_at];
#pragma unroll
        for (int j = 0; j < SPW; ++j) {
            const int k = at * kW4Block + 32 * j + col0;
            xr[j] = load8(x + (uint32_t)(xrow_at + (full ? k : min(k, d - 1))), full ? 8 : d - k);
        }
    };
    // The loaded block into LDS: x and its sums, the scales, and minus the zero points
    // (a scale times its zero point may pass fp32's range where the sum that it is
    // taken from does not).
    auto store = [&](int b) {
        unsigned char *to = smem + (b & 1) * P::X;
        vec ones;
#pragma unroll
        for (int e = 0; e < 8; ++e) ones[e] = (E)1.0f;
        constexpr int HERE = SUMS * SPW / 4, EACH = SPW / HERE;  // sums of this wavefront, steps of each
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            const float s = __uint_as_float(wr[i] & 0xffffff00u), z = (float)(wr[i] & 0xffu);
            const int at = (b & 3) * P::S + (wave * 2 + i) * GPB * 64 + word_at * 4;
            *reinterpret_cast<float *>(smem + P::S_AT + at) = s;
            *reinterpret_cast<float *>(smem + P::Z_AT + at) = -z;
        }
#pragma unroll
        for (int q = 0; q < HERE; ++q) {
            f32x4 s[2] = {{0.0f, 0.0f, 0.0f, 0.0f}, {0.0f, 0.0f, 0.0f, 0.0f}};
#pragma unroll
            for (int j = q * EACH; j < (q + 1) * EACH; ++j) {
                const RowsFrag<T> f = rows_frag<T>(xr[j]);
#pragma unroll
                for (int p = 0; p < PARTS; ++p)
                    *reinterpret_cast<vec *>(to + ((xt * 4 + step0 + j) * PARTS + p) * 1024 + lane * 16) = f.part[p];
                s[j & 1] = rows_mma_whole<T>(ones, f, s[j & 1]);
            }
            // (the same in every lane group)
            reinterpret_cast<float *>(smem + P::XS_AT + (b & 3) * P::XS)[(wave / P::XT * HERE + q) * P::ROWS + xt * 16 + lr] = s[0][0] + s[1][0];
        }
    };

    f32x4 acc[RT][MT], p[MT], sc = {0.0f, 0.0f, 0.0f, 0.0f}, zp = sc;
    float xs[MT];
    RowsFrag<T> xf[MT][STEPS];
    vec wf[STEPS];
#pragma unroll
    for (int m = 0; m < MT; ++m) {
        p[m] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
        xs[m] = 0.0f;
#pragma unroll
        for (int t = 0; t < RT; ++t) acc[t][m] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
    }
    auto read_x = [&](int b, int m, int step) {
        RowsFrag<T> f;
#pragma unroll
        for (int k = 0; k < PARTS; ++k)
            f.part[k] = *reinterpret_cast<const vec *>(smem + (b & 1) * P::X + (((wm * MT + m) * 4 + step) * PARTS + k) * 1024 + lane * 16);
        return f;
    };
    // Unit u of block b: the instructions of tile u % RT for group u / RT, and between
    // them the conversion of the next unit's weights, the sums of the unit before,
    // and behind a group's last tile the next group's x.
    auto work = [&](int b, auto number) {
        constexpr int u = decltype(number)::value, t = u % RT, q = u / RT;
        constexpr int nu = (u + 1) % UNITS, nt = nu % RT, nq = nu / RT, pt = (u + UNITS - 1) % UNITS % RT;
        if constexpr (u != 2) __builtin_amdgcn_sched_barrier(0);  // (the next block's stores go between the second's instructions)
        const int s_at = (b & 3) * P::S + ((wn * RT + t) * GPB + q) * 64 + g * 16;
        const f32x4 s_now = *reinterpret_cast<const f32x4 *>(smem + P::S_AT + s_at), z_now = *reinterpret_cast<const f32x4 *>(smem + P::Z_AT + s_at);
        float xs_now[MT];
        if constexpr (t == 0)
#pragma unroll
            for (int m = 0; m < MT; ++m) {
                const float *sums = reinterpret_cast<const float *>(smem + P::XS_AT + (b & 3) * P::XS) + (wm * MT + m) * 16 + lr;
                xs_now[m] = sums[q * SUMS / GPB * P::ROWS];
#pragma unroll
                for (int i = 1; i < SUMS / GPB; ++i) xs_now[m] += sums[(q * SUMS / GPB + i) * P::ROWS];
            }
        if constexpr (AHEAD && nq == 0) c[nt] = cr[nt];
#pragma unroll
        for (int j = 0; j < STEPS; ++j) {
#pragma unroll
            for (int m = 0; m < MT; ++m) {
                if (j == 0) {
#pragma unroll
                    for (int i = 0; i < 4; ++i) acc[pt][m][i] = fmaf(sc[i], fmaf(zp[i], xs[m], p[m][i]), acc[pt][m][i]);
                    p[m] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
                }
                p[m] = rows_mma_whole<T>(wf[j], xf[m][j], p[m]);
            }
            if constexpr (t == RT - 1)
#pragma unroll
                for (int m = 0; m < MT; ++m) xf[m][j] = read_x(u == UNITS - 1 ? b + 1 : b, m, (q + 1) % GPB * STEPS + j);
            wf[j] = w4_operand(c[nt][nq * STEPS + j], E());
        }
        sc = s_now, zp = z_now;
        if constexpr (t == 0)
#pragma unroll
            for (int m = 0; m < MT; ++m) xs[m] = xs_now[m];
        if constexpr (!AHEAD) c[nt] = load_codes(nt, nu == 0 ? b + 2 : b + 1);
        if constexpr (AHEAD && u == RT - 1)
#pragma unroll
            for (int i = 0; i < RT; ++i) cr[i] = load_codes(i, b + 1);
        // (left alone, the compiler puts the sums off to the block's end, and keeps
        // the products until then in memory)
#pragma unroll
        for (int m = 0; m < MT; ++m) asm volatile("" : "+v"(acc[pt][m]));
    };
    auto barrier = []() {
        asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
        __builtin_amdgcn_sched_barrier(0);
        __builtin_amdgcn_s_barrier();
        __builtin_amdgcn_sched_barrier(0);
    };

#pragma unroll
    for (int t = 0; t < RT; ++t) {
        c[t] = load_codes(t, 0);
        if constexpr (AHEAD) cr[t] = c[t];
    }
    load(0, std::false_type());
    store(0);
    load(1, std::false_type());
    barrier();
#pragma unroll
    for (int j = 0; j < STEPS; ++j) {
#pragma unroll
        for (int m = 0; m < MT; ++m) xf[m][j] = read_x(0, m, j);
        wf[j] = w4_operand(c[0][j], E());
    }
    if constexpr (GPB == 1) c[0] = load_codes(0, 1);
    // A block: in its second unit the next block goes to LDS, and is visible after the
    // barrier before its last unit, which reads from it.
    auto block = [&](int b, auto full) {
        each<UNITS>([&](auto number) {
            constexpr int u = decltype(number)::value;
            if constexpr (u == UNITS - 1) barrier();
            work(b, number);
            if constexpr (u == 1) {
                store(b + 1);
                load(b + 2, full);
            }
        });
    };
    int b = 0;
    for (; b + 2 < whole; ++b) block(b, std::true_type());
    for (; b < blocks; ++b) block(b, std::false_type());
#pragma unroll
    for (int m = 0; m < MT; ++m)
#pragma unroll
        for (int i = 0; i < 4; ++i) acc[RT - 1][m][i] = fmaf(sc[i], fmaf(zp[i], xs[m], p[m][i]), acc[RT - 1][m][i]);

#pragma unroll
    for (int t = 0; t < RT; t += MATS) {
        const int64_t col = (tile0 + wn * (RT / MATS) + t / MATS) * 16 + 4 * g;
        const int have = (int)max((int64_t)0, min((int64_t)4, a.f - col));
        if (have <= 0) continue;
        float bias[MATS][4];
#pragma unroll
        for (int q = 0; q < MATS; ++q)
#pragma unroll
            for (int i = 0; i < 4; ++i) bias[q][i] = a.b[q] && i < have ? a.b[q][col + i] : 0.0f;
#pragma unroll
        for (int m = 0; m < MT; ++m) {
            const int64_t row = row0 + (wm * MT + m) * 16 + lr;
            if (row >= a.n) continue;
            float v[4];
#pragma unroll
            for (int i = 0; i < 4; ++i) v[i] = acc[t][m][i] + bias[0][i];
            if constexpr (GLU)
                with_activation(a.act, [&](auto act) {
#pragma unroll
                    for (int i = 0; i < 4; ++i)
                        v[i] = activation<decltype(act)::value, sizeof(T) == 2>(v[i]) * (acc[t + MATS - 1][m][i] + bias[MATS - 1][i]);
                });
            store4((T *)a.y + row * a.f + col, have, v);
        }
    }
}

template <typename T, int GROUP, bool GLU>
hipError_t w4_tile_launch(RowsArgs a, hipStream_t st) {
    using P = W4TilePlan<T, GROUP>;
    auto kern = w4_tile_kernel<T, GROUP, GLU>;
    static std::atomic<bool> ready[kMaxDevices];  // the attribute holds for one device
    const int dev = current_device();
    if (dev < 0) return hipErrorInvalidDevice;
    if (!ready[dev].load(std::memory_order_acquire)) {
        const hipError_t e = hipFuncSetAttribute((const void *)kern, hipFuncAttributeMaxDynamicSharedMemorySize, P::LDS);
        if (e != hipSuccess) return e;
        ready[dev].store(true, std::memory_order_release);
    }
    const hipError_t e = rows_grid(a, P::ROWS, 16 * P::WN * P::RT / (GLU ? 2 : 1));
    if (e != hipSuccess) return e;
    hipLaunchKernelGGL(kern, flat_grid(rows_workgroups(a), P::THREADS), dim3(P::THREADS), P::LDS, st, a);
    return hipGetLastError();
}

}  // namespace exemcl
