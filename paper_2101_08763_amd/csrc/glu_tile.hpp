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
// A workgroup computes 256 x 256 results (8 wavefronts) or 64 x 128 (4), 64 steps of
// t a stage.  A stage of an operand is two regions in LDS, the halves that its
// wavefronts read first and second; a wavefront has 2 x 2 quarters of 16 AF x 32
// results.  Copies go from memory to LDS without registers, and what lies past
// the data reads as zeros.  B's rows are the instruction's first operand, so a
// lane's accumulators lie along a row of C.
//
// 256 x 256: a stage's 64 KiB make 128 operations a byte, so what bounds it is the
// matrix cores and the clock they leave: 16 384 x 4 096 x 8 192 x 2 of bf16 takes
// 1.59 ms, 1.38 PFLOP/s, with the matrix cores busy 74 % of the cycles at 1.9 GHz
// and no LDS conflicts (one group of wavefronts in step, where all read and then all
// multiply: 1.88 ms).  The next tile's first copies before the stores of the one
// before took 0.5 % less, tiles of 256 x 192, which fill the CUs where 256 x 256 leave a
// quarter of them idle (8 192 x 1 536 x 4 096, gradient), 2.5 %: the clock falls by
// what they gain.
// 64 x 128 fills the chip with 1/8 of the results.  A stage takes 0.45 us, of which the
// instructions are 0.12: one wavefront to a SIMD issues its copies, waits and
// multiplies in turn.  Six buffers instead of three, and reads ahead of the copies,
// changed nothing.
#pragma once

#include <algorithm>
#include <atomic>
#include <cmath>

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
    int splits;     // of the sum, over workgroups; partial: splits x pairs x M x N sums
    float *partial;
};

// Tiles: PM x PN wavefronts, quarters of 16 AF x 32 results; BUFFERS stages in LDS.
template <int AF_, int PM_, int PN_, int BUFFERS_>
struct DensePlan {
    static constexpr int AF = AF_, PM = PM_, PN = PN_, BUFFERS = BUFFERS_;
    static constexpr int WAVES = PM * PN, THREADS = WAVES * 64, BK = 64;
    static constexpr int BM = PM * 32 * AF, BN = PN * 64;
    static constexpr int A_ROWS = BM / 2, B_ROWS = BN / 2;  // of a region
    static constexpr int A_REGION = A_ROWS * BK * 2, B_REGION = B_ROWS * BK * 2;
    static constexpr int A_LOADS = A_REGION / (THREADS * 16), B_LOADS = B_REGION / (THREADS * 16);
    static constexpr int LOADS = 2 * (A_LOADS + B_LOADS);  // of a thread and stage
    static constexpr int STAGE = 2 * (A_REGION + B_REGION), LDS = BUFFERS * STAGE;
    static constexpr bool PHASED = WAVES == 8;  // two groups of wavefronts half a phase apart
    static_assert(A_LOADS >= 1 && LDS <= kLdsBytes, "geometry");
};
using LargeTile = DensePlan<4, 2, 4, 2>;  // 256 x 256
using SmallTile = DensePlan<1, 2, 2, 3>;  // 64 x 128

// Places in a region.  ALONG: a row of 8 chunks of 16 bytes (8 steps of t) per
// row of the operand; chunk c of row p is at c ^ swap(p), so that 16 rows read at
// the same chunk fill all 64 banks.  ACROSS: a row per step t with 16 bytes for 8
// rows of the operand, swapped so that the 8-byte reads of 8 rows do.
__device__ __forceinline__ int along_swap(int p) { return p >> 1 & 7; }
template <bool FIRST, int CHUNKS>
__device__ __forceinline__ int across_swap(int t) {
    if constexpr (FIRST && CHUNKS == 16) return (t & 1) | (t >> 1 & 1) << 2 | (t >> 3 & 1) << 3;
    if constexpr (FIRST) return (t >> 3 & 1) | (t >> 1 & 1) << 2;
    if constexpr (CHUNKS == 4) return (t >> 3 & 1) << 1;
    if constexpr (CHUNKS == 8) return (t >> 1 & 1) << 1 | (t >> 3 & 1) << 2;
    return (t & 3) << 1 | (t >> 3 & 1) << 3;
}

// Row of its 32 that lane lr of fragment j holds of the first operand: the four
// rows of C's accumulators i of a lane group are then 8 neighbours with those of
// the other fragment.
__device__ __forceinline__ int first_row(int lr, int j) { return 8 * (lr >> 2) + 4 * (j ^ (lr >> 2 & 1)) + (lr & 3); }

// A value that is the same in all lanes, in a scalar register.
__device__ __forceinline__ int uniform(int x) { return __builtin_amdgcn_readfirstlane(x); }
template <typename E>
__device__ __forceinline__ const E *uniform(const E *p) {
    const uint64_t v = (uint64_t)p;
    return (const E *)((uint64_t)(uint32_t)uniform((int)(v >> 32)) << 32 | (uint32_t)uniform((int)v));
}

// Eight reads of 8 bytes that transpose 4 steps of 4 x 4 rows, for two fragments of
// 16 rows x 2 x 32 steps; ROW: bytes of a step.  They are written out, with their
// wait, because the compiler waits for all copies to LDS before a transposing read.
typedef uint32_t u32x2t __attribute__((ext_vector_type(2)));
template <int ROW>
__device__ __forceinline__ void read_across(uint32_t at0, uint32_t at1, u32x2t (&v)[2][2][2]) {
    asm volatile(
        "ds_read_b64_tr_b16 %0, %8\n\t"
        "ds_read_b64_tr_b16 %1, %8 offset:%10\n\t"
        "ds_read_b64_tr_b16 %4, %9\n\t"
        "ds_read_b64_tr_b16 %5, %9 offset:%10\n\t"
        "ds_read_b64_tr_b16 %2, %8 offset:%11\n\t"
        "ds_read_b64_tr_b16 %3, %8 offset:%12\n\t"
        "ds_read_b64_tr_b16 %6, %9 offset:%11\n\t"
        "ds_read_b64_tr_b16 %7, %9 offset:%12\n\t"
        "s_waitcnt lgkmcnt(0)"
        : "=&v"(v[0][0][0]), "=&v"(v[0][0][1]), "=&v"(v[0][1][0]), "=&v"(v[0][1][1]), "=&v"(v[1][0][0]), "=&v"(v[1][0][1]),
          "=&v"(v[1][1][0]), "=&v"(v[1][1][1])
        : "v"(at0), "v"(at1), "n"(4 * ROW), "n"(32 * ROW), "n"(36 * ROW)
        : "memory");
}

// The same for one fragment.
template <int ROW>
__device__ __forceinline__ void read_across(uint32_t at, u32x2t (&v)[2][2]) {
    asm volatile(
        "ds_read_b64_tr_b16 %0, %4\n\t"
        "ds_read_b64_tr_b16 %1, %4 offset:%5\n\t"
        "ds_read_b64_tr_b16 %2, %4 offset:%6\n\t"
        "ds_read_b64_tr_b16 %3, %4 offset:%7\n\t"
        "s_waitcnt lgkmcnt(0)"
        : "=&v"(v[0][0]), "=&v"(v[0][1]), "=&v"(v[1][0]), "=&v"(v[1][1])
        : "v"(at), "n"(4 * ROW), "n"(32 * ROW), "n"(36 * ROW)
        : "memory");
}

template <typename T, int LA, int LB, int EPI, typename P>
__global__ __launch_bounds__(P::THREADS, 2) void dense_kernel(const DenseLaunch a) {
    constexpr int AF = P::AF;
    using E = typename Operand<T>::E;
    using M = Mfma<E, 16>;
    using vec = typename M::vec_t;
    constexpr int PRODUCTS = Operand<T>::PRODUCTS, BK = P::BK;
    extern __shared__ __align__(16) unsigned char smem[];
    const int tid = threadIdx.x, lane = tid & 63, lr = lane & 15, g = lane >> 4;
    const int wave = uniform(tid >> 6), wm = wave / P::PN, wn = wave % P::PN;

    // Workgroups b, b + 8, b + 16, ... share an XCD and its L2: they take
    // consecutive tiles, up to 8 of one row of tiles side by side.
    const int mblocks = a.mblocks * a.pairs, tiles = mblocks * a.nblocks, units = tiles * a.splits, per = (units + 7) / 8;
    const int wg = (int)flat_block(), pos = wg >> 3, all = (wg & 7) * per + pos;
    if (pos >= per || all >= units) return;
    const int split = uniform((uint32_t)all / (uint32_t)tiles), un = all - split * tiles;
    const int strip = uniform((uint32_t)un / (uint32_t)(mblocks * 8)), width = min(8, a.nblocks - strip * 8);
    const int in = un - strip * mblocks * 8;
    const int mt = uniform((uint32_t)in / (uint32_t)width), nt = strip * 8 + in - mt * width;
    const int other = mt >= a.mblocks ? 1 : 0;  // results of A2
    const int m0 = (mt - (other ? a.mblocks : 0)) * P::BM, n0 = nt * (EPI == GLU ? P::BN / 2 : P::BN);
    const int lda = (int)a.lda, ldb = (int)a.ldb;
    const uint32_t K = (uint32_t)a.K;  // below 2^31
    const int mrows = min(P::BM, (int)a.M - m0), nrows = min(EPI == GLU ? P::BN / 2 : P::BN, (int)a.N - n0);

    // Stages: for every pair of a matrix and a product of parts, K in steps of 64.
    // The products of small parts come first, while the sums are small.
    // A split takes a part of them.
    const int pairs = PRODUCTS * a.matrices, ksteps = (int)((K + BK - 1) / BK);
    const int each = (int)((uint32_t)(ksteps * pairs + a.splits - 1) / (uint32_t)a.splits);
    const int first = split * each, stages = max(0, min(each, ksteps * pairs - first));
    const E *at = nullptr, *bt = nullptr, *bt2 = nullptr;  // the operands of the stage to issue next
    int is_pair = uniform((uint32_t)first / (uint32_t)ksteps);
    uint32_t is_k = (uint32_t)(first - is_pair * ksteps) * BK;
    auto pair = [&]() {
        const int mat = is_pair / PRODUCTS, p = PRODUCTS - 1 - (is_pair - mat * PRODUCTS);
        const int64_t pa = PRODUCTS > 1 ? part_a(p) * a.plane_a : 0, pb = PRODUCTS > 1 ? part_b(p) * a.plane_b : 0;
        at = uniform((const E *)((mat | other) ? a.A2 : a.A) + pa + (LA == ALONG ? (int64_t)m0 * lda : m0));
        bt = uniform((const E *)(mat ? a.B2 : a.B) + pb + (LB == ALONG ? (int64_t)n0 * ldb : n0));
        if constexpr (EPI == GLU) bt2 = uniform((const E *)a.B2 + pb + (int64_t)n0 * ldb);
    };
    if (is_pair < pairs) pair();
    if constexpr (LA == ACROSS) at += (int64_t)is_k * lda;
    if constexpr (LB == ACROSS) bt += (int64_t)is_k * ldb;

    // What a thread copies of a region: a chunk of 16 bytes per load.  `off` is
    // its place in the window of the first half, `t` its first step of t.
    uint32_t a_off[P::A_LOADS], b_off[P::B_LOADS];
    uint32_t a_t[P::A_LOADS], b_t[P::B_LOADS];
#pragma unroll
    for (int i = 0; i < P::A_LOADS; ++i) {
        const int q = (wave * P::A_LOADS + i) * 64 + lane;
        if constexpr (LA == ALONG) {
            const int p = q / 8, c = (q % 8) ^ along_swap(p);
            const int row = p / (16 * AF) * (32 * AF) + p % (16 * AF);
            a_off[i] = (uint32_t)(row * lda + c * 8) * 2;
            a_t[i] = c * 8;
        } else {
            constexpr int CHUNKS = P::A_ROWS / 8;
            const int t = q / CHUNKS, e = ((q % CHUNKS) ^ across_swap<false, CHUNKS>(t)) * 8;
            const int row = e / (16 * AF) * (32 * AF) + e % (16 * AF);
            a_off[i] = (uint32_t)(t * lda + row) * 2;
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
            b_off[i] = (uint32_t)(row * ldb + c * 8) * 2;
            b_t[i] = c * 8;
        } else {
            constexpr int CHUNKS = P::B_ROWS / 8;
            const int t = q / CHUNKS, e = ((q % CHUNKS) ^ across_swap<true, CHUNKS>(t)) * 8;
            b_off[i] = (uint32_t)(t * ldb + e / 32 * APART + e % 32) * 2;
            b_t[i] = t;
        }
    }
    // Copies of half h of the stage's A or B into the buffer at `to`.  ALONG: the window
    // is the tile's rows, and a chunk past K is dead; ACROSS: it is the steps of t
    // that are left.  Past the last stage the window is empty.
    auto issue_a = [&](int h, int to) {
        uint32_t bytes = LA == ALONG ? (uint32_t)mrows * (uint32_t)lda * 2 : (min((uint32_t)BK, K - is_k) * (uint32_t)lda - (uint32_t)m0) * 2;
        if (is_pair >= pairs) bytes = 0;
        const auto win = window_rsrc(at, bytes);
#pragma unroll
        for (int i = 0; i < P::A_LOADS; ++i) {
            uint32_t off = a_off[i] + (uint32_t)(LA == ALONG ? h * 16 * AF * lda * 2 + is_k * 2 : h * 16 * AF * 2);
            if constexpr (LA == ALONG) off = is_k + a_t[i] < K ? off : kDeadOffset;
            window_to_lds16(win, smem + to + h * P::A_REGION + (wave * P::A_LOADS + i) * 1024, off);
        }
    };
    auto issue_b = [&](int h, int to) {
        uint32_t bytes = LB == ALONG ? (uint32_t)nrows * (uint32_t)ldb * 2 : (min((uint32_t)BK, K - is_k) * (uint32_t)ldb - (uint32_t)n0) * 2;
        if (is_pair >= pairs) bytes = 0;
        const auto win = window_rsrc(EPI == GLU && h ? bt2 : bt, bytes);
        const int half = EPI == GLU ? 0 : h;
#pragma unroll
        for (int i = 0; i < P::B_LOADS; ++i) {
            uint32_t off = b_off[i] + (uint32_t)(LB == ALONG ? half * 32 * ldb * 2 + is_k * 2 : half * 32 * 2);
            if constexpr (LB == ALONG) off = is_k + b_t[i] < K ? off : kDeadOffset;
            window_to_lds16(win, smem + to + 2 * P::A_REGION + h * P::B_REGION + (wave * P::B_LOADS + i) * 1024, off);
        }
    };
    auto issued = [&]() {
        is_k += BK;
        if constexpr (LA == ACROSS) at += (int64_t)BK * lda;
        if constexpr (LB == ACROSS) bt += (int64_t)BK * ldb;
        if (is_k >= K) {
            is_k = 0;
            if (++is_pair < pairs) pair();
        }
    };

    // Operands of one half from LDS, fragments of 16 rows x 32 steps.
    const uint32_t lds = (uint32_t)(uintptr_t)(__attribute__((address_space(3))) unsigned char *)smem;
    auto join = [](u32x2t lo, u32x2t hi) { return __builtin_bit_cast(vec, u32x4{lo[0], lo[1], hi[0], hi[1]}); };
    auto read_a = [&](int h, int from, vec(&av)[AF][2]) {  // [fragment][32 steps]
        const int region = from + h * P::A_REGION;
        if constexpr (LA == ALONG) {
#pragma unroll
            for (int ks = 0; ks < 2; ++ks)
#pragma unroll
                for (int w = 0; w < AF; ++w) {
                    const int p = wm * 16 * AF + w * 16 + lr;
                    av[w][ks] = *reinterpret_cast<const vec *>(smem + region + p * 128 + ((ks * 4 + g) ^ along_swap(lr)) * 16);
                }
        } else {
            constexpr int CHUNKS = P::A_ROWS / 8;
            const int t = 8 * g + (lr >> 2);
            auto place = [&](int w) {
                const int c = wm * 2 * AF + w * 2 + (lr >> 1 & 1);
                return lds + region + t * CHUNKS * 16 + (c ^ across_swap<false, CHUNKS>(t)) * 16 + (lr & 1) * 8;
            };
            if constexpr (AF == 1) {
                u32x2t v[2][2];
                read_across<CHUNKS * 16>(place(0), v);
#pragma unroll
                for (int ks = 0; ks < 2; ++ks) av[0][ks] = join(v[ks][0], v[ks][1]);
            } else {
#pragma unroll
                for (int w = 0; w < AF; w += 2) {
                    u32x2t v[2][2][2];
                    read_across<CHUNKS * 16>(place(w), place(w + 1), v);
#pragma unroll
                    for (int e = 0; e < 2; ++e)
#pragma unroll
                        for (int ks = 0; ks < 2; ++ks) av[w + e][ks] = join(v[e][ks][0], v[e][ks][1]);
                }
            }
        }
    };
    auto read_b = [&](int h, int from, vec(&to)[2][2]) {
        const int region = from + 2 * P::A_REGION + h * P::B_REGION;
        if constexpr (LB == ALONG) {
#pragma unroll
            for (int ks = 0; ks < 2; ++ks)
#pragma unroll
                for (int j = 0; j < 2; ++j) {
                    const int p = wn * 32 + j * 16 + lr;
                    to[j][ks] = *reinterpret_cast<const vec *>(smem + region + p * 128 + ((ks * 4 + g) ^ along_swap(lr)) * 16);
                }
        } else {
            constexpr int CHUNKS = P::B_ROWS / 8;
            const int t = 8 * g + (lr >> 2), c = wn * 4 + (lr & 3);
            const uint32_t at = lds + region + t * CHUNKS * 16 + (c ^ across_swap<true, CHUNKS>(t)) * 16 + (lr & 1) * 8;
            u32x2t v[2][2][2];
            read_across<CHUNKS * 16>(at, at ^ 8, v);
#pragma unroll
            for (int j = 0; j < 2; ++j)
#pragma unroll
                for (int ks = 0; ks < 2; ++ks) to[j][ks] = join(v[j][ks][0], v[j][ks][1]);
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

    auto multiply = [&](int ha, int hb, const vec(&av)[AF][2], const vec(&b)[2][2]) {
#pragma unroll
        for (int ks = 0; ks < 2; ++ks)
#pragma unroll
            for (int w = 0; w < AF; ++w)
#pragma unroll
                for (int j = 0; j < 2; ++j) acc[ha][w][hb][j] = M::mma(b[j][ks], av[w][ks], 0, acc[ha][w][hb][j]);
    };
    auto issue = [&](int to) {
        issue_b(0, to);
        issue_a(0, to);
        issue_b(1, to);
        issue_a(1, to);
        issued();
    };
    if constexpr (P::PHASED) {
        // A phase: reads for one quarter of the tile and copies for the stage that
        // comes into this buffer next, then the quarter's instructions.  The
        // wavefronts 0 .. 3 are half a phase ahead of 4 .. 7, with which they share the
        // SIMDs: while one reads, the other multiplies.  What is read in a phase has
        // been waited for, by every wavefront, in the one before it; the copies go to
        // the region that was read there.
        vec av[AF][2], bv[3][2][2];  // B's second half, and the first one's of two stages
        // (two regions of the stage before, and whole stages)
        constexpr int FLYING = P::LOADS / 2 + (P::BUFFERS - 1) * P::LOADS;
        auto ready = [&]() {
            asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)" ::"n"(FLYING) : "memory");
            __builtin_amdgcn_sched_barrier(0);
            __builtin_amdgcn_s_barrier();
            __builtin_amdgcn_sched_barrier(0);
        };
        auto quarter = [&](int ha, int hb, const vec(&b)[2][2]) {
            __builtin_amdgcn_s_setprio(1);
            multiply(ha, hb, av, b);
            __builtin_amdgcn_s_setprio(0);
            __builtin_amdgcn_sched_barrier(0);
            __builtin_amdgcn_s_barrier();
            __builtin_amdgcn_sched_barrier(0);
        };
        static_assert(P::BUFFERS == 2, "the buffer is a constant of each stage");
        auto stage = [&](auto parity) {
            constexpr int own = 1 + decltype(parity)::value, others = 3 - own;
            constexpr int at = decltype(parity)::value * P::STAGE, other_at = P::STAGE - at;
            read_a(0, at, av);
            issue_b(0, at);
            ready();
            quarter(0, 0, bv[own]);
            read_b(1, at, bv[0]);
            issue_a(0, at);
            ready();
            quarter(0, 1, bv[0]);
            read_a(1, at, av);
            issue_b(1, at);
            ready();
            quarter(1, 1, bv[0]);
            read_b(0, other_at, bv[others]);
            issue_a(1, at);
            issued();
            ready();
            quarter(1, 0, bv[own]);
        };
#pragma unroll
        for (int buf = 0; buf < P::BUFFERS; ++buf) issue(buf * P::STAGE);
        ready();
        read_b(0, 0, bv[1]);
        asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
        __builtin_amdgcn_sched_barrier(0);
        __builtin_amdgcn_s_barrier();
        if (wave >= 4) __builtin_amdgcn_s_barrier();
        __builtin_amdgcn_sched_barrier(0);
        for (int st = 0; st < stages; st += 2) {
            stage(std::integral_constant<int, 0>());
            if (st + 1 < stages) stage(std::integral_constant<int, 1>());
        }
        if (wave < 4) __builtin_amdgcn_s_barrier();
    } else {
        // Two such workgroups share a CU, and each covers the other's waits.
#pragma unroll
        for (int buf = 0; buf < P::BUFFERS - 1; ++buf) issue(buf * P::STAGE);
        auto next = [](int at) { return at == (P::BUFFERS - 1) * P::STAGE ? 0 : at + P::STAGE; };
        int at = 0, to = (P::BUFFERS - 1) * P::STAGE;
        for (int st = 0; st < stages; ++st) {
            // (__syncthreads would wait for all copies)
            asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)" ::"n"((P::BUFFERS - 2) * P::LOADS) : "memory");  // stage st
            __builtin_amdgcn_sched_barrier(0);
            __builtin_amdgcn_s_barrier();  // everyone's, and the one before it has been read
            __builtin_amdgcn_sched_barrier(0);
            issue(to);
            vec av[2][AF][2], bv[2][2][2];
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                read_b(h, at, bv[h]);
                read_a(h, at, av[h]);
            }
#pragma unroll
            for (int ha = 0; ha < 2; ++ha)
#pragma unroll
                for (int hb = 0; hb < 2; ++hb) multiply(ha, hb, av[ha], bv[hb]);
            to = at;
            at = next(at);
        }
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
        auto store_to = [&](auto *C) {
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
        };
        if (a.splits == 1)
            store_to((T *)(other ? a.C2 : a.C));
        else
            store_to(a.partial + ((int64_t)split * a.pairs + other) * a.M * a.N);
    }
}

// out = the splits' sums, added in their order.  Bound by reading them (they are
// written just before: from the caches; 4.9 us for 2 x 777 x 301, of which most is the
// launch).
template <typename T>
__global__ __launch_bounds__(256) void dense_join_kernel(const float *__restrict__ partial, int splits, int64_t count,
                                                         int64_t of_one, T *__restrict__ C, T *__restrict__ C2) {
    const int64_t at = (flat_block() * 256 + threadIdx.x) * 4;
    if (at >= count) return;
    const int have = (int)min((int64_t)4, count - at);
    typedef float vec __attribute__((ext_vector_type(4), aligned(4)));
    float s[4] = {};
    for (int i = 0; i < splits; ++i) {
        const float *p = partial + i * count + at;
        if (have == 4) {
            const vec v = *reinterpret_cast<const vec *>(p);
#pragma unroll
            for (int e = 0; e < 4; ++e) s[e] += v[e];
        } else {
#pragma unroll
            for (int e = 0; e < 3; ++e)
                if (e < have) s[e] += p[e];
        }
    }
    if (at + have <= of_one) {
        store4(C + at, have, s);
    } else if (at >= of_one) {
        store4(C2 + (at - of_one), have, s);
    } else {
#pragma unroll
        for (int e = 0; e < 4; ++e)
            if (e < have) (at + e < of_one ? C[at + e] : C2[at + e - of_one]) = (T)s[e];
    }
}

template <typename T, int LA, int LB, int EPI, typename P>
hipError_t dense_launch(DenseLaunch a, hipStream_t st) {
    auto kern = dense_kernel<T, LA, LB, EPI, P>;
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
    if (mb * a.pairs * a.splits > (int64_t(1) << 30) / nb) return hipErrorInvalidValue;
    a.mblocks = (int)mb;
    a.nblocks = (int)nb;
    hipLaunchKernelGGL(kern, flat_grid((mb * a.pairs * a.splits * nb + 7) / 8 * 8, P::THREADS), dim3(P::THREADS), P::LDS, st, a);
    return hipGetLastError();
}

// Tiles and splits for a product of M x N (pairs times), `stages` steps long, by an
// estimate: 1.4 us a stage of the large tiles and 0.45 of the small ones, rounds of
// workgroups over the CUs (one to a CU, also of the small ones, of which two fit: a stage's
// time is that of a CU with one), and for splits of the sum their fp32 values written and
// read.  Measured, us, small and large tiles: block of bf16 100 x 1 536 x 4 096 14 / 33,
// 2 000 x 1 536 x 4 096 70 / 45, 8 192 x 1 536 x 4 096 260 / 162, of fp32 128 x 1 024 x 2 048
// 54 / 125; gradient of bf16 1 000 x 1 536 x 4 096 105 / 196, 8 192 x 1 536 x 4 096 906 / 412.
// Without and with splits: gradient of bf16 16 000 x 128 x 512 130 / 46, of fp32 2 000 x
// 2 048 x 4 096 1 274 / 704.
struct DenseChoice {
    bool large;
    int splits;
    double us;
};
inline DenseChoice dense_choice(int64_t M, int64_t N, int64_t pairs, int64_t stages, bool glu, bool may_split) {
    const double cus = (double)std::max<int64_t>(1, device_cu_count());
    const int64_t half = glu ? 2 : 1;
    DenseChoice best{false, 1, 0.0};
    for (const bool large : {false, true}) {
        const int64_t bm = large ? LargeTile::BM : SmallTile::BM, bn = (large ? LargeTile::BN : SmallTile::BN) / half;
        const double tiles = (double)(((M + bm - 1) / bm) * ((N + bn - 1) / bn) * pairs);
        for (int64_t s = 1; s <= 32 && s <= stages; s = s < 4 ? s + 1 : s + s / 4) {
            if (s > 1 && (!may_split || (double)s * (double)(pairs * M * N) > 2.5e8)) break;
            const double each = (double)((stages + s - 1) / s);
            double t = std::max(1.0, std::ceil(tiles * (double)s / cus)) * (large ? 1.4 * each + 6.0 : 0.45 * each + 3.0);
            if (s > 1) t += 4.0 + 2.2e-6 * (double)(s * pairs * M * N);
            if (best.us == 0.0 || t < best.us) best = {large, (int)s, t};
        }
    }
    return best;
}

template <typename T, int LA, int LB, int EPI>
hipError_t dense_run(DenseLaunch a, hipStream_t st) {
    const int64_t stages = (a.K + 63) / 64 * Operand<T>::PRODUCTS * a.matrices;
    const DenseChoice c = dense_choice(a.M, a.N, a.pairs, stages, EPI == GLU, a.partial != nullptr);
    a.splits = c.splits;
    const hipError_t e = c.large ? dense_launch<T, LA, LB, EPI, LargeTile>(a, st) : dense_launch<T, LA, LB, EPI, SmallTile>(a, st);
    if (e != hipSuccess || c.splits == 1) return e;
    const int64_t of_one = a.M * a.N, count = of_one * a.pairs;
    hipLaunchKernelGGL(dense_join_kernel<T>, flat_grid((count + 1023) / 1024, 256), dim3(256), 0, st, a.partial, c.splits,
                       count, of_one, (T *)a.C, (T *)a.C2);
    return hipGetLastError();
}

// Bytes of the splits' sums.
template <typename T>
int64_t dense_partial_bytes(int64_t M, int64_t N, int64_t K, int64_t pairs, int64_t matrices) {
    const DenseChoice c = dense_choice(M, N, pairs, (K + 63) / 64 * Operand<T>::PRODUCTS * matrices, false, true);
    return c.splits == 1 ? 0 : c.splits * pairs * M * N * 4;
}

inline DenseLaunch dense_args(const DenseArgs &a) {
    DenseLaunch l{};
    l.A = a.A.p, l.A2 = a.A.p2, l.B = a.B.p, l.B2 = a.B.p2;
    l.lda = a.A.ld, l.ldb = a.B.ld, l.plane_a = a.A.plane, l.plane_b = a.B.plane;
    l.M = a.M, l.N = a.N, l.K = a.K;
    l.matrices = 1, l.pairs = 1;
    l.bg = a.bg, l.bu = a.bu, l.act = a.act;
    l.C = a.C, l.C2 = a.C2, l.g = a.g, l.u = a.u;
    l.splits = 1, l.partial = a.partial;
    return l;
}

}  // namespace exemcl
