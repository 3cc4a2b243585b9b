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
// coordinates go to the wavefronts in turn, whose sums are added in order.  For
// results too few to fill the chip with larger tiles: 1 x 20 000 x 1 536 takes 7
// us (2.4 TB/s), a launch and the wait for three loads in turn.
constexpr int kDirectWaves = 4;

template <typename T, int BITS_A>
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
            i32x8 high, low;
            mx_divide(a, high, low);
            acc = mx_mma(b, low, acc, sb, sa);
            acc = mx_mma(b, high, acc, sb, sa);
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
// Tiles of C through LDS.  PM x PN wavefronts compute (16 WM PM) x (64 NB PN)
// elements, one K-step of 128 coordinates a stage, DEPTH stages in LDS.  B's
// rows are the instruction's first operand, so a lane's accumulators lie along
// a row of C, 16 bytes of fp32 results.  For 16-bit ones fragment j of a block of
// 64 holds B's rows 4 i + j (i = 0 .. 15), which makes them 16 neighbours and a
// wavefront's stores whole 128-byte lines; A's are dealt out the same way (row
// WM i + w in fragment w).
// Copies run along the rows, 4 or 8 lanes to one (a lane per row, the operands'
// own order, takes the address units 64 steps a load instead of 16: 16 384 x
// 8 192 x 4 096 565 us).
//
// That size, 8 by 4 bits to bf16, takes 662 us: two instructions for every 128
// coordinates (mx_divide), together at 3.3 PFLOP/s where the instruction alone, on
// random values, runs at 4.2; the matrix cores are busy 75 % of the time.  4 by 4
// bits takes 312 (3.5 of 6.8).  The rest is the start and the end of a tile, LDS
// reads and copies between instructions, and the clock, which the chip lowers on
// random values.
// ---------------------------------------------------------------------------
template <int BITS_A, int WM, int NB, int PM, int PN, int DEPTH>
struct MxTilePlan {
    static constexpr int WAVES = PM * PN, THREADS = WAVES * 64, BM = PM * WM * 16, BN = PN * NB * 64;
    static constexpr int A_FRAGS = PM * WM * BITS_A / 4, B_FRAGS = PN * NB * 4;  // of 1 KiB
    static constexpr int A_LOADS = A_FRAGS / WAVES, B_LOADS = B_FRAGS / WAVES;
    static constexpr int LOADS = A_LOADS + B_LOADS;  // per thread and stage, beside the scales
    static constexpr int S_LOADS = (BM + BN + THREADS - 1) / THREADS;
    // 16-byte chunks of a row in a stage, 4 or 8 (4- or 8-bit rows); chunk c of
    // row p goes to place c ^ swap(p).  The 16 rows that lanes read the same
    // chunk of then fill all 64 banks once, and so do 8 such rows and the 8
    // others of the next chunk.  (The conflicts that are counted, two cycles for
    // each, are those of the scales' byte reads.)
    static constexpr int A_CHUNKS = BITS_A;
    template <int CHUNKS>
    __device__ __forceinline__ static int swap(int p) {
        if constexpr (CHUNKS == 8) return ((p >> 2 ^ p >> 3) & 1) << 2 | (p >> 3 & 1) << 1 | (p >> 1 & 1);
        return ((p >> 2 ^ p >> 3) & 1) << 1 | (p >> 3 & 1);
    }
    static constexpr int B_AT = A_FRAGS * 1024, BUF = B_AT + B_FRAGS * 1024;
    static constexpr int SCALES_AT = DEPTH * BUF, SBUF = S_LOADS * THREADS * 16, LDS = SCALES_AT + 2 * SBUF;
    static_assert(A_FRAGS % WAVES == 0 && B_FRAGS % WAVES == 0 && BM % 64 == 0 && LDS <= kLdsBytes, "geometry");
};

template <typename T, int BITS_A, int WM, int NB, int PM, int PN, int DEPTH>
__global__ __launch_bounds__(PM *PN * 64, 2) void mx_product_kernel(
    const uint8_t *__restrict__ A, const uint8_t *__restrict__ As, int64_t m, const uint8_t *__restrict__ B,
    const uint8_t *__restrict__ Bs, int64_t n, int ksteps, int mblocks, int nblocks, const float *__restrict__ bias,
    T *__restrict__ C) {
    using P = MxTilePlan<BITS_A, WM, NB, PM, PN, DEPTH>;
    constexpr int WN = 4 * NB, H = BITS_A / 4;  // fragments of B, halves of one of A's
    extern __shared__ __align__(16) unsigned char smem[];
    const int tid = threadIdx.x, lane = tid & 63, lr = lane & 15, g = lane >> 4;
    const int wave = __builtin_amdgcn_readfirstlane(tid >> 6), wm = wave % PM, wn = wave / PM;

    // Workgroups b, b + 8, b + 16, ... share an XCD and its L2: they take
    // consecutive tiles, up to 8 of one row of tiles side by side.
    const int64_t units = (int64_t)mblocks * nblocks, per = (units + 7) / 8;
    const int64_t wg = flat_block(), pos = wg >> 3, u = (wg & 7) * per + pos;
    if (pos >= per || u >= units) return;
    const int64_t strip = u / ((int64_t)mblocks * 8);
    const int width = (int)min((int64_t)8, nblocks - strip * 8);
    const int64_t in = u - strip * mblocks * 8;
    const int64_t m0 = in / width * P::BM, n0 = (strip * 8 + in % width) * P::BN;

    // What a thread copies: its part of A's and B's fragments, and the scales of
    // 64 rows.  What lies past the rows, or in stages past the last, reads as
    // zeros.
    const int a_row = ksteps * 16 * BITS_A, b_row = ksteps * 64, s_row = ksteps * 4;
    const uint32_t mrows = (uint32_t)min((int64_t)P::BM, m - m0), nrows = (uint32_t)min((int64_t)P::BN, n - n0);
    const auto awin = window_rsrc(A + m0 * a_row, mrows * (uint32_t)a_row);
    const auto bwin = window_rsrc(B + n0 * b_row, nrows * (uint32_t)b_row);
    const auto aswin = window_rsrc(As + m0 * s_row, mrows * (uint32_t)s_row);
    const auto bswin = window_rsrc(Bs + n0 * s_row, nrows * (uint32_t)s_row);
    // Copy i takes A's places 64 (wave A_LOADS + i) ... in LDS order.  Which rows
    // those are differs between copies by a number that is the same for all
    // lanes, up to the parity of i, where a row has 8 chunks.
    auto b_row_at = [](int p) { return sizeof(T) == 4 ? p : p / 64 * 64 + p % 16 * 4 + p / 16 % 4; };
    uint32_t a_off[2], b_off;
    int a_more[P::A_LOADS], b_more[P::B_LOADS];
    auto a_place = [&](int i, int at, int &row, int &c) {
        const int p = ((wave * P::A_LOADS + i) * 64 + at) / P::A_CHUNKS;
        row = p / (WM * 16) * (WM * 16) + p % 16 * WM + p / 16 % WM;
        c = at % P::A_CHUNKS ^ P::template swap<P::A_CHUNKS>(p);
    };
    auto b_place = [&](int i, int at, int &row, int &c) {
        const int p = ((wave * P::B_LOADS + i) * 64 + at) / 4;
        row = b_row_at(p);
        c = at % 4 ^ P::template swap<4>(p);
    };
#pragma unroll
    for (int i = 0; i < P::A_LOADS; ++i) {
        int row, c, row0, c0;
        a_place(i, lane, row, c);
        if (i < 2) a_off[i] = (uint32_t)(row * a_row + c * 16);
        a_place(i, 0, row, c);
        a_place(i % 2, 0, row0, c0);
        a_more[i] = (row - row0) * a_row;
    }
#pragma unroll
    for (int i = 0; i < P::B_LOADS; ++i) {
        int row, c, row0, c0;
        b_place(i, lane, row, c);
        if (i == 0) b_off = (uint32_t)(row * b_row + c * 16);
        b_place(i, 0, row, c);
        b_place(0, 0, row0, c0);
        b_more[i] = (row - row0) * b_row;
    }
    // (in LDS the scales of a fragment's 16 rows are neighbours)
    uint32_t s_off[P::S_LOADS];
#pragma unroll
    for (int i = 0; i < P::S_LOADS; ++i) {
        const int p = i * P::THREADS + tid, q = p - P::BM;
        s_off[i] = (uint32_t)((p < P::BM ? p / (WM * 16) * (WM * 16) + p % 16 * WM + p / 16 % WM
                                         : b_row_at(q)) * s_row);
    }
    // Copy number i of stage st (A's first) into the buffer at `to`.
    auto copy = [&](int st, int to, int i) {
        const uint32_t dead = st < ksteps ? 0u : kDeadOffset;
        if (i < P::A_LOADS)
            window_to_lds16(awin, smem + to + (wave * P::A_LOADS + i) * 1024,
                            a_off[i % 2] + (dead | (uint32_t)(a_more[i] + st * 16 * BITS_A)));
        else
            window_to_lds16(bwin, smem + to + P::B_AT + (wave * P::B_LOADS + i - P::A_LOADS) * 1024,
                            b_off + (dead | (uint32_t)(b_more[i - P::A_LOADS] + st * 64)));
    };
    auto copy_scales = [&](int st) {
        if (st % 4 != 0) return;
        const uint32_t dead = (st < ksteps ? 0u : kDeadOffset) | (uint32_t)(st * 4);
        unsigned char *buf = smem + P::SCALES_AT + st / 4 % 2 * P::SBUF;
#pragma unroll
        for (int i = 0; i < P::S_LOADS; ++i) {
            const int p = i * P::THREADS + wave * 64;
            if (P::BM % P::THREADS == 0 ? i * P::THREADS < P::BM : p < P::BM)
                window_to_lds16(aswin, buf + p * 16, s_off[i] + dead);
            else
                window_to_lds16(bswin, buf + p * 16, s_off[i] + dead);
        }
    };
    auto issue = [&](int st) {
        copy_scales(st);
#pragma unroll
        for (int i = 0; i < P::LOADS; ++i) copy(st, st * P::BUF, i);
    };

    f32x4 acc[WM][WN];
#pragma unroll
    for (int w = 0; w < WM; ++w)
#pragma unroll
        for (int j = 0; j < WN; ++j) acc[w][j] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};

    // A stage's operands are read from LDS while the stage before it computes,
    // each over the one just used for the last time.  Only the copies then stand
    // between a barrier and the next instructions.
    i32x4 b[WN];
    int bs[WN];
    i32x4 a[WM][H];
    int as[WM];
    int a_at[H];
#pragma unroll
    for (int h = 0; h < H; ++h)
        a_at[h] = (wm * WM * 16 + lr) * P::A_CHUNKS * 16 + ((h * 4 + g) ^ P::template swap<P::A_CHUNKS>(lr)) * 16;
    const int b_at = P::B_AT + (wn * NB * 64 + lr) * 64 + (g ^ P::template swap<4>(lr)) * 16;
    const int s_at = P::SCALES_AT + lr * 16 + g;
    // Where a stage's operands are: one register each, so that the reads differ
    // by constants.
    struct Places {
        int a[H], b, as, bs;
    };
    auto places = [&](int st, int from) {
        Places x;
#pragma unroll
        for (int h = 0; h < H; ++h) {
            x.a[h] = from + a_at[h];
            asm("" : "+v"(x.a[h]));
        }
        x.b = from + b_at;
        x.as = s_at + st / 4 % 2 * P::SBUF + st % 4 * 4 + wm * WM * 256;
        x.bs = s_at + st / 4 % 2 * P::SBUF + st % 4 * 4 + (P::BM + wn * WN * 16) * 16;
        asm("" : "+v"(x.b), "+v"(x.as), "+v"(x.bs));
        return x;
    };
    auto read_a = [&](const Places &x, int w) {
#pragma unroll
        for (int h = 0; h < H; ++h) a[w][h] = *reinterpret_cast<const i32x4 *>(smem + x.a[h] + w * P::A_CHUNKS * 256);
        as[w] = smem[x.as + w * 256];
    };
    auto read_b = [&](const Places &x, int j) {
        b[j] = *reinterpret_cast<const i32x4 *>(smem + x.b + j * 1024);
        bs[j] = smem[x.bs + j * 256];
    };
    // Stage st; the next one is in LDS at `from`, and this one's place `to` is
    // free for st + DEPTH.
    auto stage = [&](int st, int from, int to) {
        asm volatile("s_waitcnt vmcnt(%0)" ::"n"((DEPTH - 2) * P::LOADS) : "memory");  // stage st + 1
        __syncthreads();                                               // everyone's, and st has been read
        copy_scales(st + DEPTH);
        __builtin_amdgcn_sched_barrier(0);
        const Places x = places(st + 1, from);
#pragma unroll
        for (int w = 0; w < WM; ++w) {
            if (w > 0) read_a(x, w - 1);
#pragma unroll
            for (int i = w * P::LOADS / WM; i < (w + 1) * P::LOADS / WM; ++i) copy(st + DEPTH, to, i);
            if constexpr (BITS_A == 4) {
#pragma unroll
                for (int j = 0; j < WN; ++j) {
                    acc[w][j] = mx_mma(b[j], a[w][0], acc[w][j], bs[j], as[w]);
                    if (w == WM - 1) read_b(x, j);
                }
            } else {
                i32x8 high, low;
                mx_divide(mx_join(a[w][0], a[w][1]), high, low);
#pragma unroll
                for (int j = 0; j < WN; ++j) acc[w][j] = mx_mma(b[j], low, acc[w][j], bs[j], as[w]);
#pragma unroll
                for (int j = 0; j < WN; ++j) {
                    acc[w][j] = mx_mma(b[j], high, acc[w][j], bs[j], as[w]);
                    if (w == WM - 1) read_b(x, j);
                }
            }
            // Reads and copies between the instructions: all at once, they hold
            // the wavefront up for as long as LDS and the address units take
            // them in.
#pragma unroll
            for (int i = 0; i < H + 1; ++i) {
                __builtin_amdgcn_sched_group_barrier(0x100, 1, 0);
                __builtin_amdgcn_sched_group_barrier(0x008, 1, 0);
            }
#pragma unroll
            for (int i = 0; i < (P::LOADS + WM - 1) / WM; ++i) {
                __builtin_amdgcn_sched_group_barrier(0x020, 1, 0);
                __builtin_amdgcn_sched_group_barrier(0x008, 1, 0);
            }
            if (w == WM - 1) {
#pragma unroll
                for (int i = 0; i < WN; ++i) {
                    __builtin_amdgcn_sched_group_barrier(0x100, 2, 0);
                    __builtin_amdgcn_sched_group_barrier(0x008, 1, 0);
                }
            }
            __builtin_amdgcn_sched_group_barrier(0x008, WN * 2, 0);
            __builtin_amdgcn_sched_barrier(0);
        }
        read_a(x, WM - 1);
    };

#pragma unroll
    for (int st = 0; st < DEPTH; ++st) issue(st);
    asm volatile("s_waitcnt vmcnt(%0)" ::"n"((DEPTH - 1) * P::LOADS) : "memory");
    __syncthreads();
    {
        const Places x = places(0, 0);
#pragma unroll
        for (int w = 0; w < WM; ++w) read_a(x, w);
#pragma unroll
        for (int j = 0; j < WN; ++j) read_b(x, j);
    }
    for (int st = 0, at = 0; st < ksteps; ++st) {
        const int from = at == (DEPTH - 1) * P::BUF ? 0 : at + P::BUF;
        stage(st, from, at);
        at = from;
    }
    asm volatile("s_waitcnt vmcnt(0)" ::: "memory");  // the last copies

    // Accumulator i of fragment j of a block of 64 is its column 16 g + 4 i + j;
    // with 32-bit results 16 j + 4 g + i.
#pragma unroll
    for (int q = 0; q < NB; ++q) {
        const int64_t block = n0 + (wn * NB + q) * 64;
        if constexpr (sizeof(T) == 4) {
            typedef float vec __attribute__((ext_vector_type(4), aligned(4)));
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                const int64_t col = block + j * 16 + g * 4;
                const int have = (int)max((int64_t)0, min((int64_t)4, n - col));
                f32x4 bb;
#pragma unroll
                for (int e = 0; e < 4; ++e) bb[e] = bias && e < have ? bias[col + e] : 0.0f;
#pragma unroll
                for (int w = 0; w < WM; ++w) {
                    const int64_t row = m0 + wm * WM * 16 + lr * WM + w;
                    const f32x4 v = acc[w][q * 4 + j] + bb;
                    if (row >= m) continue;
                    float *c = (float *)C + row * n + col;
                    if (have == 4) {
                        *reinterpret_cast<vec *>(c) = v;
                    } else {
#pragma unroll
                        for (int e = 0; e < 3; ++e)
                            if (e < have) c[e] = v[e];
                    }
                }
            }
        } else {
            const int64_t col = block + g * 16;
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
                    lo[e] = acc[w][q * 4 + e % 4][e / 4] + bb[e];
                    hi[e] = acc[w][q * 4 + e % 4][e / 4 + 2] + bb[e + 8];
                }
                if (row < m) {
                    T *c = C + row * n + col;
                    store8(c, have, lo);
                    store8(c + 8, have - 8, hi);
                }
            }
        }
    }
}

template <typename T, int BITS_A>
hipError_t product_direct(const MxProductArgs &a, hipStream_t st) {
    const int64_t mt = (a.m + 15) / 16, nt = (a.n + 15) / 16;
    if (mt > (int64_t(1) << 34) / nt) return hipErrorInvalidValue;  // 2^14 rows of kFlatRow
    hipLaunchKernelGGL((mx_product_direct_kernel<T, BITS_A>), flat_grid(mt * nt, kDirectWaves * 64),
                       dim3(kDirectWaves * 64), 0, st, (const uint8_t *)a.A, (const uint8_t *)a.A_scales, a.m,
                       (const uint8_t *)a.B, (const uint8_t *)a.B_scales, a.n, a.d, nt, a.bias, (T *)a.C);
    return hipGetLastError();
}

template <typename T, int BITS_A, int WM, int NB, int PM, int PN, int DEPTH>
hipError_t product_tiled(const MxProductArgs &a, hipStream_t st) {
    using P = MxTilePlan<BITS_A, WM, NB, PM, PN, DEPTH>;
    auto kern = mx_product_kernel<T, BITS_A, WM, NB, PM, PN, DEPTH>;
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

// The kernel for a size.  16 x 16 tiles, with the coordinates dealt out to four
// wavefronts, where a fitted time says that they take less than tiles of 64 x 128:
// mostly up to 16 rows; else the largest tile that still makes enough of them (us,
// to bf16; 8 and 4: bits of A):
//                            16x16  64x128  128x128  128x256  256x256
//   1 x 28 672 x 8 192     8  36.6    65.0
//                          4  35.3    35.5
//   8 x 28 672 x 8 192     8  51.9    66.1
//                          4  45.0    36.3
//   8 x 20 000 x 1 536     8   8.5    16.5     17.0     23.6
//                          4   7.1     9.0      9.3     14.5
//   24 x 2 000 x 1 024     8   3.7    12.1     12.6     17.4
//                          4   3.4     7.2      7.3     10.6
//   130 x 8 192 x 1 024    8  23.3    12.6     13.2     18.7     30.0
//                          4  19.6     7.6      8.5     12.3     12.8
//   1 024 x 8 192 x 1 024  8          32.9     20.7     21.0     32.3
//                          4          16.3     12.3     14.7     16.1
//   1 024 x 30 000 x 1 024 8         102       68.5     56.4     70.3
//                          4          50.6     38.4     39.9     40.8
//   16 384 x 8 192 x 1 024 8         407      247      188      253
//                          4         163      116      123      129
//   16 384 x 8 192 x 4 096 8        1394      818      654      805
//                          4         506      408      354      312
// The largest has one workgroup per CU, which starts and ends alone: with 4-bit
// rows it wins from about 1 500 coordinates on, where its last round is full; with
// 8-bit rows two workgroups per CU cover the division, and it never does.
// Stores of fp32 results overlap less of what follows them, and 128 x 256 pays
// earlier (333 x 30 011 x 301 of 8 bits, 2.75 tiles of 128 x 128 a CU: 21.2 us
// instead of 22.9).  With 4-bit rows two stages are enough for 128 x 128 and let
// three workgroups share a CU (the same to bf16: 12.8 us instead of 16.2).
template <typename T, int BITS_A>
hipError_t product_run(const MxProductArgs &a, hipStream_t st) {
    const int64_t cus = std::max<int64_t>(1, device_cu_count());
    auto tiles = [&](int64_t bm, int64_t bn) { return ((a.m + bm - 1) / bm) * ((a.n + bn - 1) / bn); };
    const double ks = (double)(mx_padded(a.d) / kMxRow);
    // us, fitted to 1 to 512 x 2 000 to 50 000 x 256 to 8 192.  A tile of 16 x 16
    // takes half its time for B and half for the rows of A that there are; tiles of
    // 64 x 128 two to a CU half of what they take one after the other.
    const double rows = 0.5 * (double)((a.m + 15) / 16) + (double)a.m / 32.0;
    const double direct = 2.6 + 0.06 * ks + (BITS_A == 8 ? 4.6e-4 : 3.8e-4) * rows * (double)((a.n + 15) / 16) * (ks + 0.5);
    const double tiled = (5.8 + (BITS_A == 8 ? 0.9 : 0.3) * ks) * (1.0 + (double)std::max<int64_t>(0, tiles(64, 128) - cus) / (2.0 * cus));
    if (direct <= tiled) return product_direct<T, BITS_A>(a, st);
    if (tiles(64, 128) <= cus) return product_tiled<T, BITS_A, 4, 1, 1, 2, 3>(a, st);
    if (tiles(128, 128) * 2 <= (sizeof(T) == 4 ? 5 : 6) * cus)
        return product_tiled<T, BITS_A, 4, 1, 2, 2, BITS_A == 8 ? 3 : 2>(a, st);
    if constexpr (BITS_A == 4) {
        const int64_t large = tiles(256, 256), last = (large + cus - 1) / cus * cus;
        if (ks >= 12 && last * 10 <= large * 11) return product_tiled<T, BITS_A, 8, 1, 2, 4, 3>(a, st);
    }
    return product_tiled<T, BITS_A, 4, 2, 2, 2, 2>(a, st);
}

template <int BITS_A>
hipError_t product_typed(int prec, const MxProductArgs &a, hipStream_t st) {
    if (prec == P_FP32) return product_run<float, BITS_A>(a, st);
    if (prec == P_FP16) return product_run<_Float16, BITS_A>(a, st);
    return product_run<__bf16, BITS_A>(a, st);
}

}  // namespace exemcl
