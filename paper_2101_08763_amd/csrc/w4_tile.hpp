// w4_tile.hpp -- products by 4-bit weights and the gated block on them for many
// rows (instantiated in kernels_w4_*.hip).
//
// The arithmetic is that of glu_rows.hpp: instructions on whole numbers q, the sum
// of a group's x beside them, scale and zero point applied in fp32 once per group.
// Here a workgroup of 8 wavefronts computes 128 rows of x by 256 weights' rows (GLU:
// 128 of each matrix), 128 coordinates a stage.  Wavefront w loads the 16 rows of x
// that are tile w, which is operand order: its registers go to LDS as they are
// (fp32: in parts, made once) and to one instruction on ones for the sums.  A
// wavefront has 4 x 4 tiles of results; its weights come from memory, a stage ahead,
// and are converted once for four tiles of x.
#pragma once

#include <atomic>

#include "glu_rows.hpp"

namespace exemcl {

template <typename T, int GROUP>
struct W4TilePlan {
    static constexpr int WAVES = 8, THREADS = WAVES * 64, RT = 4, MT = 4, WN = 4;
    static constexpr int PARTS = Operand<T>::PARTS, BUFFERS = PARTS == 1 ? 2 : 1;
    static constexpr int GPB = kW4Block / GROUP, STEPS = GROUP / 32;
    static constexpr int X = WAVES * 4 * PARTS * 1024;       // bytes of x in a stage
    static constexpr int XS = GPB * WAVES * 16 * 4;          // its groups' sums
    static constexpr int WORDS = WN * RT * GPB * 64;         // the weights' words
    static constexpr int XS_AT = BUFFERS * X, WORDS_AT = XS_AT + 2 * XS, LDS = WORDS_AT + 2 * WORDS;
    static_assert(LDS <= kLdsBytes, "geometry");
};

template <typename T, int GROUP, bool GLU>
__global__ __launch_bounds__(512, 2) void w4_tile_kernel(const RowsArgs a) {
    using P = W4TilePlan<T, GROUP>;
    using E = typename Operand<T>::E;
    using vec = typename Mfma<E, 16>::vec_t;
    constexpr int RT = P::RT, MT = P::MT, GPB = P::GPB, STEPS = P::STEPS, PARTS = P::PARTS, MATS = GLU ? 2 : 1;
    extern __shared__ __align__(16) unsigned char smem[];
    const int lane = threadIdx.x & 63, lr = lane & 15, g = lane >> 4;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), wm = wave & 1, wn = wave >> 1;

    // Workgroups b, b + 8, ... share an XCD and its L2: blocks of rows that read the
    // same weights follow each other there.
    const int64_t wg = flat_block(), pos = wg >> 3, unit = pos / a.mblocks * 8 + (wg & 7), mb = pos % a.mblocks;
    if (unit >= a.units) return;
    const int64_t d = a.d, row0 = mb * 128, tile0 = unit * (P::WN * RT / MATS), ftiles = (a.f + 15) / 16;
    const int blocks = (int)w4_blocks(d), whole = (int)(d / kW4Block);

    const T *x = (const T *)a.x + min(row0 + wave * 16 + lr, a.n - 1) * d + 8 * g;
    // Tile t of this wavefront (GLU: gate and up in turn), past the last one it again.
    auto tile_of = [&](int wn, int t) { return min(tile0 + wn * (RT / MATS) + t / MATS, ftiles - 1); };
    const u32x4 *codes[RT];
#pragma unroll
    for (int t = 0; t < RT; ++t) codes[t] = (const u32x4 *)a.w[t % MATS] + tile_of(wn, t) * blocks * 64 + lane;
    // Words: wavefront w < WN GPB / 4 copies 64 lanes' 16 bytes, 4 to a group of a tile.
    constexpr int WORD_WAVES = P::WORDS / 1024;
    const u32x4 *words;
    {
        const int q = (wave % WORD_WAVES) * 16 + (lane >> 2), t = q / GPB;
        words = (const u32x4 *)a.words[t % RT % MATS] + (tile_of(t / RT, t % RT) * blocks * GPB + q % GPB) * 4 + (lane & 3);
    }

    typename Chunk<T>::vec xr[4];
    u32x4 cr[RT], c[RT], wr;
    auto load = [&](int b) {
        const int at = min(b, blocks - 1);  // past the last block it again, never used
#pragma unroll
        for (int t = 0; t < RT; ++t) cr[t] = codes[t][at * 64];
        if (wave < WORD_WAVES) wr = words[at * GPB * 4];
        if (at < whole) {
#pragma unroll
            for (int j = 0; j < 4; ++j) xr[j] = load8(x + at * kW4Block + 32 * j, 8);
        } else {
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                const int k = at * kW4Block + 32 * j;
                xr[j] = load8(x + min((int64_t)k, d - 1 - 8 * g), (int)(d - 8 * g - k));
            }
        }
    };
    // The loaded block into LDS.
    auto store = [&](int b) {
        unsigned char *to = smem + b % P::BUFFERS * P::X;
        vec ones;
#pragma unroll
        for (int e = 0; e < 8; ++e) ones[e] = (E)1.0f;
#pragma unroll
        for (int q = 0; q < GPB; ++q) {
            f32x4 s = {0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
            for (int j = q * STEPS; j < (q + 1) * STEPS; ++j) {
                const RowsFrag<T> f = rows_frag<T>(xr[j]);
#pragma unroll
                for (int p = 0; p < PARTS; ++p)
                    *reinterpret_cast<vec *>(to + ((wave * 4 + j) * PARTS + p) * 1024 + lane * 16) = f.part[p];
                s = rows_mma_whole<T>(ones, f, s);
            }
            if (g == 0) reinterpret_cast<float *>(smem + P::XS_AT + (b & 1) * P::XS)[q * 128 + wave * 16 + lr] = s[0];
        }
        if (wave < WORD_WAVES)
            *reinterpret_cast<u32x4 *>(smem + P::WORDS_AT + (b & 1) * P::WORDS + wave * 1024 + lane * 16) = wr;
    };

    f32x4 acc[RT][MT];
#pragma unroll
    for (int t = 0; t < RT; ++t)
#pragma unroll
        for (int m = 0; m < MT; ++m) acc[t][m] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};

    load(0);
    store(0);
#pragma unroll
    for (int t = 0; t < RT; ++t) c[t] = cr[t];
    __syncthreads();
    for (int b = 0; b < blocks; ++b) {
        load(b + 1);
        const unsigned char *from = smem + b % P::BUFFERS * P::X + wm * MT * 4 * PARTS * 1024 + lane * 16;
        const float *sums = reinterpret_cast<const float *>(smem + P::XS_AT + (b & 1) * P::XS) + wm * MT * 16 + lr;
        const unsigned char *scales = smem + P::WORDS_AT + (b & 1) * P::WORDS + wn * RT * GPB * 64 + g * 16;
#pragma unroll
        for (int q = 0; q < GPB; ++q) {
            RowsFrag<T> xf[PARTS == 1 ? MT : 1][STEPS];
            float xs[MT];
#pragma unroll
            for (int m = 0; m < MT; ++m) xs[m] = sums[q * 128 + m * 16];
            auto fragment = [&](int m, int j) {
                RowsFrag<T> f;
#pragma unroll
                for (int p = 0; p < PARTS; ++p)
                    f.part[p] = *reinterpret_cast<const vec *>(from + ((m * 4 + q * STEPS + j) * PARTS + p) * 1024);
                return f;
            };
            if constexpr (PARTS == 1)
#pragma unroll
                for (int m = 0; m < MT; ++m)
#pragma unroll
                    for (int j = 0; j < STEPS; ++j) xf[m][j] = fragment(m, j);
#pragma unroll
            for (int t = 0; t < RT; ++t) {
                const u32x4 word = *reinterpret_cast<const u32x4 *>(scales + (t * GPB + q) * 64);
                vec wf[STEPS];
#pragma unroll
                for (int j = 0; j < STEPS; ++j) wf[j] = w4_operand(c[t][q * STEPS + j], E());
                f32x4 p[MT];
#pragma unroll
                for (int m = 0; m < MT; ++m) p[m] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
                for (int j = 0; j < STEPS; ++j)
#pragma unroll
                    for (int m = 0; m < MT; ++m)
                        p[m] = rows_mma_whole<T>(wf[j], PARTS == 1 ? xf[PARTS == 1 ? m : 0][j] : fragment(m, j), p[m]);
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    const float s = __uint_as_float(word[i] & 0xffffff00u), z = -(float)(word[i] & 0xffu);
#pragma unroll
                    for (int m = 0; m < MT; ++m) acc[t][m][i] = fmaf(s, fmaf(z, xs[m], p[m][i]), acc[t][m][i]);
                }
                if (PARTS > 1 && t + 1 < RT) __builtin_amdgcn_sched_barrier(0);
            }
            // (left alone, the compiler puts these sums off to the stage's end, and
            // keeps each group's products until then in memory)
#pragma unroll
            for (int t = 0; t < RT; ++t)
#pragma unroll
                for (int m = 0; m < MT; ++m) asm volatile("" : "+v"(acc[t][m]));
            __builtin_amdgcn_sched_barrier(0);
        }
        if (P::BUFFERS == 1) __syncthreads();  // everyone has read this block
        store(b + 1);
#pragma unroll
        for (int t = 0; t < RT; ++t) c[t] = cr[t];
        __syncthreads();
    }

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
    const int64_t tiles = P::WN * P::RT / (GLU ? 2 : 1);
    a.mblocks = (a.n + 127) / 128;
    a.units = ((a.f + 15) / 16 + tiles - 1) / tiles;
    const int64_t groups = (a.units + 7) / 8;
    if (groups > (int64_t(1) << 31) / a.mblocks) return hipErrorInvalidValue;
    hipLaunchKernelGGL(kern, flat_grid(groups * 8 * a.mblocks, P::THREADS), dim3(P::THREADS), P::LDS, st, a);
    return hipGetLastError();
}

}  // namespace exemcl
