// glu_tile.hpp -- tiled products for the gated block on many rows and for its
// gradient (instantiated in kernels_glu_{forward,dx,dw}*.hip).
//
//   C[i][j] = sum_t A(i, t) B(j, t)
//
// where an operand lies in memory along t (ALONG: x and the weights in the forward
// pass, dg and du in dx) or across it (ACROSS: the weights in dx; dg, du and x in
// dw), with up to twelve pairs of operands added up: the two matrices of dx, and
// the six products of fp32's parts.
//
// A workgroup of 8 wavefronts computes 64 AF x 256 results, 64 steps of t a
// stage.  A stage of an operand is two regions in LDS, the halves that its
// wavefronts read first and second; a wavefront has 2 x 2 quarters of 16 AF x 32
// results.  Copies go from memory to LDS without registers, and what lies past
// the data reads as zeros.  B's rows are the instruction's first operand, so a
// lane's accumulators lie along a row of C.
#pragma once

#include <algorithm>
#include <atomic>

#include "glu_device.hpp"
#include "mfma_kernels.hpp"

namespace exemcl {

enum DenseLayout { ALONG = 0, ACROSS = 1 };
enum DenseEpilogue { STORE = 0, GLU = 1 };

struct DenseLaunch {
    const void *A, *A2, *B, *B2;
    int64_t lda, ldb, plane_a, plane_b;
    int64_t M, N, K;
    int matrices;            // of the sum (dx: 2)
    int mblocks, nblocks;
    int pairs;               // results of A and of A2 apart (dw)
    const float *bg, *bu;
    int act;
    void *C, *C2, *g, *u;
};

template <int AF>
struct DensePlan {
    static constexpr int WAVES = 8, THREADS = WAVES * 64, BK = 64;
    static constexpr int BM = 64 * AF, BN = 256;
    static constexpr int A_ROWS = BM / 2, B_ROWS = BN / 2;  // of a region
    static constexpr int A_REGION = A_ROWS * BK * 2, B_REGION = B_ROWS * BK * 2;
    static constexpr int A_LOADS = A_REGION / (THREADS * 16), B_LOADS = B_REGION / (THREADS * 16);
    static constexpr int STAGE = 2 * (A_REGION + B_REGION), LDS = 2 * STAGE;
    static_assert(A_LOADS >= 1 && LDS <= kLdsBytes, "geometry");
};

// Places in a region.  ALONG: a row of 8 chunks of 16 bytes (8 steps of t) per
// row of the operand; chunk c of row p is at c ^ swap(p), so that 16 rows read at
// the same chunk fill all 64 banks.  ACROSS: a row per step t with 16 bytes for 8
// rows of the operand, swapped so that the 8-byte reads of 8 rows do.
__device__ __forceinline__ int along_swap(int p) { return p >> 1 & 7; }
template <bool FIRST, int CHUNKS>
__device__ __forceinline__ int across_swap(int t) {
    if constexpr (FIRST) return (t & 1) | (t >> 1 & 1) << 2 | (t >> 3 & 1) << 3;
    if constexpr (CHUNKS == 8) return (t >> 1 & 1) << 1 | (t >> 3 & 1) << 2;
    return (t & 3) << 1 | (t >> 3 & 1) << 3;
}

// Row of its 32 that lane lr of fragment j holds of the first operand: the four
// rows of C's accumulators i of a lane group are then 8 neighbours with those of
// the other fragment.
__device__ __forceinline__ int first_row(int lr, int j) { return 8 * (lr >> 2) + 4 * (j ^ (lr >> 2 & 1)) + (lr & 3); }

template <typename T, int LA, int LB, int EPI, int AF>
__global__ __launch_bounds__(512, 2) void dense_kernel(const DenseLaunch a) {
    using P = DensePlan<AF>;
    using E = typename Operand<T>::E;
    using M = Mfma<E, 16>;
    using vec = typename M::vec_t;
    constexpr int PRODUCTS = Operand<T>::PRODUCTS, BK = P::BK;
    extern __shared__ __align__(16) unsigned char smem[];
    const int tid = threadIdx.x, lane = tid & 63, lr = lane & 15, g = lane >> 4;
    const int wave = __builtin_amdgcn_readfirstlane(tid >> 6), wm = wave >> 2, wn = wave & 3;

    // Workgroups b, b + 8, b + 16, ... share an XCD and its L2: they take
    // consecutive tiles, up to 8 of one row of tiles side by side.
    const int64_t mblocks = (int64_t)a.mblocks * a.pairs, units = mblocks * a.nblocks, per = (units + 7) / 8;
    const int64_t wg = flat_block(), pos = wg >> 3, un = (wg & 7) * per + pos;
    if (pos >= per || un >= units) return;
    const int64_t strip = un / (mblocks * 8);
    const int width = (int)min((int64_t)8, a.nblocks - strip * 8);
    const int64_t in = un - strip * mblocks * 8;
    const int64_t mt = in / width;
    const bool other = mt >= a.mblocks;  // results of A2
    const int64_t m0 = (mt - (other ? a.mblocks : 0)) * P::BM;
    const int64_t n0 = (strip * 8 + in % width) * (EPI == GLU ? P::BN / 2 : P::BN);

    // Stages: for every matrix and product of parts, K in steps of 64.
    const int ksteps = (int)((a.K + BK - 1) / BK), stages = ksteps * PRODUCTS * a.matrices;
    const E *at, *bt, *bt2;  // the pair's operands, from this tile's rows on
    auto pair = [&](int s) {
        const int mat = s / PRODUCTS, p = s - mat * PRODUCTS;
        at = (const E *)((mat | (int)other) ? a.A2 : a.A) + (PRODUCTS > 1 ? part_a(p) * a.plane_a : 0);
        bt = (const E *)(mat ? a.B2 : a.B) + (PRODUCTS > 1 ? part_b(p) * a.plane_b : 0);
        at += LA == ALONG ? m0 * a.lda : m0;
        if constexpr (EPI == GLU) bt2 = (const E *)a.B2 + (PRODUCTS > 1 ? part_b(p) * a.plane_b : 0) + n0 * a.ldb;
        bt += LB == ALONG ? n0 * a.ldb : n0;
    };
    pair(0);
    int is_pair = 0, is_k = 0;  // the stage to issue next

    // What a thread copies of a region: a chunk of 16 bytes per load.  `off` is
    // its place in the window of the first half, `t` its first step of t.
    uint32_t a_off[P::A_LOADS], b_off[P::B_LOADS];
    int a_t[P::A_LOADS], b_t[P::B_LOADS];
#pragma unroll
    for (int i = 0; i < P::A_LOADS; ++i) {
        const int q = (wave * P::A_LOADS + i) * 64 + lane;
        if constexpr (LA == ALONG) {
            const int p = q / 8, c = (q % 8) ^ along_swap(p);
            const int row = p / (16 * AF) * (32 * AF) + p % (16 * AF);
            a_off[i] = (uint32_t)(row * (int)a.lda + c * 8) * 2;
            a_t[i] = c * 8;
        } else {
            constexpr int CHUNKS = P::A_ROWS / 8;
            const int t = q / CHUNKS, e = ((q % CHUNKS) ^ across_swap<false, CHUNKS>(t)) * 8;
            const int row = e / (16 * AF) * (32 * AF) + e % (16 * AF);
            a_off[i] = (uint32_t)(t * (int)a.lda + row) * 2;
            a_t[i] = t;
        }
    }
#pragma unroll
    for (int i = 0; i < P::B_LOADS; ++i) {
        const int q = (wave * P::B_LOADS + i) * 64 + lane;
        constexpr int APART = EPI == GLU ? 32 : 64;  // from one wavefront's columns to the next one's
        if constexpr (LB == ALONG) {
            const int p = q / 8, c = (q % 8) ^ along_swap(p);
            const int row = p / 32 * APART + first_row(p % 16, p / 16 % 2);
            b_off[i] = (uint32_t)(row * (int)a.ldb + c * 8) * 2;
            b_t[i] = c * 8;
        } else {
            const int t = q / 16, e = ((q % 16) ^ across_swap<true, 16>(t)) * 8;
            b_off[i] = (uint32_t)(t * (int)a.ldb + e / 32 * APART + e % 32) * 2;
            b_t[i] = t;
        }
    }
    // Copies of half h of a stage's A or B into the buffer at `to`.  ALONG: the
    // window is the tile's rows, and a chunk past K is dead; ACROSS: it is the
    // steps of t that are left.
    auto issue_a = [&](int h, int to) {
        const int64_t k0 = (int64_t)is_k * BK;
        const bool live = is_pair < PRODUCTS * a.matrices;
        const E *base = LA == ALONG ? at : at + k0 * a.lda;
        const int64_t rows = LA == ALONG ? min((int64_t)P::BM, a.M - m0) : min((int64_t)BK, a.K - k0);
        const int64_t bytes = (rows * a.lda - (LA == ALONG ? 0 : m0)) * 2;
        const auto win = window_rsrc(base, live ? (uint32_t)max((int64_t)0, bytes) : 0u);
#pragma unroll
        for (int i = 0; i < P::A_LOADS; ++i) {
            uint32_t off = a_off[i];
            if constexpr (LA == ALONG)
                off = k0 + a_t[i] < a.K ? off + (uint32_t)(k0 * 2) + (uint32_t)(h * 16 * AF * (int)a.lda * 2) : kDeadOffset;
            else
                off += h * 16 * AF * 2;
            window_to_lds16(win, smem + to + h * P::A_REGION + (wave * P::A_LOADS + i) * 1024, off);
        }
    };
    auto issue_b = [&](int h, int to) {
        const int64_t k0 = (int64_t)is_k * BK;
        const bool live = is_pair < PRODUCTS * a.matrices;
        const E *base = EPI == GLU && h ? bt2 : LB == ALONG ? bt : bt + k0 * a.ldb;
        const int64_t rows = LB == ALONG ? min((int64_t)(EPI == GLU ? P::BN / 2 : P::BN), a.N - n0) : min((int64_t)BK, a.K - k0);
        const int64_t bytes = (rows * a.ldb - (LB == ALONG ? 0 : n0)) * 2;
        const auto win = window_rsrc(base, live ? (uint32_t)max((int64_t)0, bytes) : 0u);
#pragma unroll
        for (int i = 0; i < P::B_LOADS; ++i) {
            uint32_t off = b_off[i];
            const int half = EPI == GLU ? 0 : h;
            if constexpr (LB == ALONG)
                off = k0 + b_t[i] < a.K ? off + (uint32_t)(k0 * 2) + (uint32_t)(half * 32 * (int)a.ldb * 2) : kDeadOffset;
            else
                off += half * 32 * 2;
            window_to_lds16(win, smem + to + 2 * P::A_REGION + h * P::B_REGION + (wave * P::B_LOADS + i) * 1024, off);
        }
    };
    auto issued = [&]() {
        if (++is_k == ksteps) {
            is_k = 0;
            if (++is_pair < PRODUCTS * a.matrices) pair(is_pair);
        }
    };

    // Operands of one half from LDS, fragments of 16 rows x 32 steps.
    typedef __attribute__((address_space(3))) i16x4 lds_i16x4;
    auto across = [&](int byte, int row_bytes) {
        const auto lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_i16x4 *)(smem + byte));
        const auto hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_i16x4 *)(smem + byte + 4 * row_bytes));
        return __builtin_bit_cast(vec, __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7));
    };
    vec av[AF][2], bv[2][2][2];  // [fragment][step]; B's of both halves
    auto read_a = [&](int h, int from) {
        const int region = from + h * P::A_REGION;
#pragma unroll
        for (int w = 0; w < AF; ++w)
#pragma unroll
            for (int ks = 0; ks < 2; ++ks) {
                if constexpr (LA == ALONG) {
                    const int p = wm * 16 * AF + w * 16 + lr;
                    av[w][ks] = *reinterpret_cast<const vec *>(smem + region + p * 128 + ((ks * 4 + g) ^ along_swap(lr)) * 16);
                } else {
                    constexpr int CHUNKS = P::A_ROWS / 8;
                    const int t = ks * 32 + 8 * g + (lr >> 2), c = wm * 2 * AF + w * 2 + (lr >> 1 & 1);
                    av[w][ks] = across(region + t * CHUNKS * 16 + (c ^ across_swap<false, CHUNKS>(t)) * 16 + (lr & 1) * 8, CHUNKS * 16);
                }
            }
    };
    auto read_b = [&](int h, int from) {
        const int region = from + 2 * P::A_REGION + h * P::B_REGION;
#pragma unroll
        for (int j = 0; j < 2; ++j)
#pragma unroll
            for (int ks = 0; ks < 2; ++ks) {
                if constexpr (LB == ALONG) {
                    const int p = wn * 32 + j * 16 + lr;
                    bv[h][j][ks] = *reinterpret_cast<const vec *>(smem + region + p * 128 + ((ks * 4 + g) ^ along_swap(lr)) * 16);
                } else {
                    const int t = ks * 32 + 8 * g + (lr >> 2), c = wn * 4 + (lr & 3);
                    bv[h][j][ks] = across(region + t * 256 + (c ^ across_swap<true, 16>(t)) * 16 + (j ^ (lr & 1)) * 8, 256);
                }
            }
    };
    f32x4 acc[2][AF][2][2];
#pragma unroll
    for (int ha = 0; ha < 2; ++ha)
#pragma unroll
        for (int w = 0; w < AF; ++w)
#pragma unroll
            for (int hb = 0; hb < 2; ++hb)
#pragma unroll
                for (int j = 0; j < 2; ++j) acc[ha][w][hb][j] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
    auto multiply = [&](int ha, int hb) {
#pragma unroll
        for (int ks = 0; ks < 2; ++ks)
#pragma unroll
            for (int w = 0; w < AF; ++w)
#pragma unroll
                for (int j = 0; j < 2; ++j) acc[ha][w][hb][j] = M::mma(bv[hb][j][ks], av[w][ks], 0, acc[ha][w][hb][j]);
    };

    auto issue = [&](int to) {
        issue_a(0, to);
        issue_b(0, to);
        issue_b(1, to);
        issue_a(1, to);
        issued();
    };
    issue(0);
    for (int st = 0; st < stages; ++st) {
        const int from = (st & 1) * P::STAGE;
        asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
        __syncthreads();
        issue(P::STAGE - from);
        read_a(0, from);
        read_b(0, from);
        read_b(1, from);
        multiply(0, 0);
        multiply(0, 1);
        read_a(1, from);
        multiply(1, 0);
        multiply(1, 1);
    }
    asm volatile("s_waitcnt vmcnt(0)" ::: "memory");  // the last copies

    // Row w * 16 + lr of a quarter, and its columns 8 g .. 8 g + 7: fragment g % 2
    // first.
    auto eight = [&](const f32x4(&v)[2], float(&o)[8]) {
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            o[i] = g & 1 ? v[1][i] : v[0][i];
            o[i + 4] = g & 1 ? v[0][i] : v[1][i];
        }
    };
    if constexpr (EPI == GLU) {
        const int64_t col = n0 + wn * 32 + 8 * g;
        const int have = (int)max((int64_t)0, min((int64_t)8, a.N - col));
        float bias[2][8];
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            bias[0][i] = a.bg && i < have ? a.bg[col + i] : 0.0f;
            bias[1][i] = a.bu && i < have ? a.bu[col + i] : 0.0f;
        }
        with_activation(a.act, [&](auto act) {
#pragma unroll
            for (int ha = 0; ha < 2; ++ha)
#pragma unroll
                for (int w = 0; w < AF; ++w) {
                    const int64_t row = m0 + wm * 32 * AF + ha * 16 * AF + w * 16 + lr;
                    if (row >= a.M) continue;
                    float gv[8], uv[8], hv[8];
                    eight(acc[ha][w][0], gv);
                    eight(acc[ha][w][1], uv);
#pragma unroll
                    for (int i = 0; i < 8; ++i) {
                        gv[i] += bias[0][i];
                        uv[i] += bias[1][i];
                        hv[i] = activation<decltype(act)::value, sizeof(T) == 2>(gv[i]) * uv[i];
                    }
                    const int64_t to = row * a.N + col;
                    store8((T *)a.C + to, have, hv);
                    if (a.g) store8((T *)a.g + to, have, gv);
                    if (a.u) store8((T *)a.u + to, have, uv);
                }
        });
    } else {
        T *C = (T *)(other ? a.C2 : a.C);
#pragma unroll
        for (int ha = 0; ha < 2; ++ha)
#pragma unroll
            for (int w = 0; w < AF; ++w) {
                const int64_t row = m0 + wm * 32 * AF + ha * 16 * AF + w * 16 + lr;
                if (row >= a.M) continue;
#pragma unroll
                for (int hb = 0; hb < 2; ++hb) {
                    const int64_t col = n0 + wn * 64 + hb * 32 + 8 * g;
                    const int have = (int)max((int64_t)0, min((int64_t)8, a.N - col));
                    float v[8];
                    eight(acc[ha][w][hb], v);
                    store8(C + row * a.N + col, have, v);
                }
            }
    }
}

template <typename T, int LA, int LB, int EPI, int AF>
hipError_t dense_launch(DenseLaunch a, hipStream_t st) {
    using P = DensePlan<AF>;
    auto kern = dense_kernel<T, LA, LB, EPI, AF>;
    static std::atomic<bool> ready[kMaxDevices];  // the attribute holds for one device
    const int dev = current_device();
    if (dev < 0) return hipErrorInvalidDevice;
    if (!ready[dev].load(std::memory_order_acquire)) {
        const hipError_t e = hipFuncSetAttribute((const void *)kern, hipFuncAttributeMaxDynamicSharedMemorySize, P::LDS);
        if (e != hipSuccess) return e;
        ready[dev].store(true, std::memory_order_release);
    }
    constexpr int BN = EPI == GLU ? P::BN / 2 : P::BN;
    const int64_t mb = (a.M + P::BM - 1) / P::BM, nb = (a.N + BN - 1) / BN;
    if (mb * a.pairs > (int64_t(1) << 30) / nb) return hipErrorInvalidValue;
    a.mblocks = (int)mb;
    a.nblocks = (int)nb;
    hipLaunchKernelGGL(kern, flat_grid((mb * a.pairs * nb + 7) / 8 * 8, P::THREADS), dim3(P::THREADS), P::LDS, st, a);
    return hipGetLastError();
}

// The kernel for a size: 256 x 256 tiles.
template <typename T, int LA, int LB, int EPI>
hipError_t dense_run(const DenseLaunch &a, hipStream_t st) {
    const int64_t cus = std::max<int64_t>(1, device_cu_count());
    const int64_t bn = EPI == GLU ? 128 : 256;
    if (((a.M + 255) / 256) * a.pairs * ((a.N + bn - 1) / bn) >= cus) return dense_launch<T, LA, LB, EPI, 4>(a, st);
    return dense_launch<T, LA, LB, EPI, 2>(a, st);
}

inline DenseLaunch dense_args(const DenseArgs &a) {
    DenseLaunch l{};
    l.A = a.A.p, l.A2 = a.A.p2, l.B = a.B.p, l.B2 = a.B.p2;
    l.lda = a.A.ld, l.ldb = a.B.ld, l.plane_a = a.A.plane, l.plane_b = a.B.plane;
    l.M = a.M, l.N = a.N, l.K = a.K;
    l.matrices = 1, l.pairs = 1;
    l.bg = a.bg, l.bu = a.bu, l.act = a.act;
    l.C = a.C, l.C2 = a.C2, l.g = a.g, l.u = a.u;
    return l;
}

}  // namespace exemcl
