// mx_sets.hpp -- f(S) = (2/n) sum_v max(0, max_s <v, s> - |s|^2 / 2) on 4-bit
// rows: the clamp form of mfma_kernels.hpp on the 4-bit matrix cores, whose
// sums of products are exact in fp32 (instantiated in kernels_mx_sets_*.hip).
//
// A workgroup keeps WAVES x RT x 16 points in registers (4 of them hold 16
// points x 128 coordinates, a quarter of what 16-bit rows take) and the set
// members stream past them through LDS: a tile is one member of each of 16
// sets, two tiles a unit, UPS units a stage, three stages in flight.  A lane's
// column is one set, so the maximum over its members stays in a register until
// the set group ends.  Rows past n read as zeros and add nothing, a bias being
// at most 0.  A sum of every 32 points is written, in the same order whatever
// RT and WAVES are, so these follow the launch and not the result.
//
// What bounds it is the matrix cores: 512 sets of 32 on 200 000 x 256 take 335 us
// (5.0 PFLOP/s; the instruction alone, on random values, runs at 6.8), 512 of 16
// on 20 000 x 1 536 119.  Two workgroups of 4 wavefronts to a CU beat one of 8,
// which meets at a barrier every stage (200 000 x 256: 396 us when the smaller
// ones took 361; 100 000 x 1 024, 512 of 16: 400 against 340); above 1 024
// coordinates, where two row tiles are all that fit beside 10 or more fragments
// each, LDS has room for one workgroup, and one of 8 wavefronts covers its LDS
// reads better (100 000 x 1 536, 256 of 16: 329 us; one wavefront to a SIMD with
// four row tiles 332, and 163 against 147 at 1 792).
#pragma once

#include <float.h>

#include <algorithm>
#include <atomic>
#include <type_traits>
#include <utility>

#include "internal.h"
#include "mfma_kernels.hpp"
#include "mx_device.hpp"

namespace exemcl {

constexpr int kMxSetRows = 32;        // points per partial sum
constexpr int64_t kMxSetsD = 2048;    // longest rows kept in registers
constexpr int64_t kMxGatherUnits = 8; // pairs of members a workgroup stages itself
// Members of a set, and pairs of members a workgroup goes through, that the
// kernels count in 32 bits (the tiles of one group of so many take a terabyte).
constexpr int64_t kMxMembers = int64_t(1) << 30;

// Arguments of one launch: tiles (or biases) go to `work`.
struct MxSetsArgs {
    const uint8_t *codes, *scales;
    int64_t n, d;
    const int32_t *sets;
    int64_t l, k;
    uint8_t *work;
    float *partials;
    int64_t lpad;
};

hipError_t mx_sets_short(int ks, const MxSetsArgs &x, hipStream_t st);
hipError_t mx_sets_wide(int ks, const MxSetsArgs &x, hipStream_t st);

// A tile: KS fragments of 1 KiB in operand order, per 4 of them the scales of
// every lane (byte b: of fragment 4 q + b), and 16 biases -|s|^2 / 2 (-FLT_MAX:
// no member).
template <int KS>
struct MxTile {
    static constexpr int SCALES = KS * 1024, BIAS = SCALES + (KS + 3) / 4 * 256, BYTES = BIAS + 64;
};

template <typename F, int... I>
__device__ __forceinline__ void each_step(F f, std::integer_sequence<int, I...>) {
    (f(std::integral_constant<int, I>{}), ...);
}

template <int KS, int RT, int WAVES>
struct MxSetsPlan {
    static constexpr int UNIT = 2 * MxTile<KS>::BYTES, THREADS = WAVES * 64;
    static constexpr int UPS = UNIT >= 16384 ? 1 : 16384 / UNIT;            // units per stage
    static constexpr int STAGE = UPS * UNIT;
    static constexpr int LOADS = (STAGE + THREADS * 16 - 1) / (THREADS * 16);  // per thread
    // The operands of a tile are read while the one before it computes, each over
    // the one just used: 100 000 x 1 536, 256 sets of 16 329 us instead of 354,
    // 50 000 x 768, 512 of 16 142 (150), 200 000 x 256, 512 of 32 346 (360).  Not
    // for one fragment a tile (3 % slower), nor for four with 8 row tiles, which
    // leave no registers (184 us instead of 110).
    static constexpr bool AHEAD = WAVES > 4 || (RT > 2 && KS != 1 && KS != 4);
    static constexpr int DEPTH = AHEAD ? 4 : 3, BUF = LOADS * THREADS * 16, LDS = DEPTH * BUF;
    static constexpr int ROWS = WAVES * RT * 16;
    static_assert(LDS <= kLdsBytes && RT % 2 == 0, "geometry");
};

// One tile, member p of the 16 sets of group grp, by WPT wavefronts of a
// workgroup that take turns of four fragments (WPT = 1: any one wavefront).
// |s|^2 in 64 bits (the squares of a block's elements add up to a whole number
// of quarters); `part`: LDS, 16 doubles a wavefront.  `there` false: nothing is
// read or written.
template <int KS, int WPT>
__device__ __forceinline__ void mx_pack_tile(const uint8_t *__restrict__ codes, const uint8_t *__restrict__ scales, int64_t n,
                                             int ksteps, const int32_t *__restrict__ sets, int64_t l, int k, int64_t grp,
                                             int p, bool there, uint8_t *t, double (*part)[16]) {
    using T = MxTile<KS>;
    const int wave = threadIdx.x >> 6, turn = wave % WPT, lane = threadIdx.x & 63, lr = lane & 15, g = lane >> 4;
    const int64_t j = grp * 16 + lr;
    const int64_t s = there ? sets[min(j, l - 1) * k + p] : -1;
    const bool live = there && j < l && s >= 0 && s < n;
    const int64_t row = live ? s : 0;
    double q = 0.0;
    if (there) {
#pragma unroll
        for (int r0 = 0; r0 < (KS + 3) / 4; r0 += WPT) {
            const int r = r0 + turn;
            uint32_t packed = 0;
#pragma unroll
            for (int b = 0; b < 4; ++b) {
                const int ks = r * 4 + b;
                if (ks >= KS) break;
                i32x4 x = {0, 0, 0, 0};
                uint32_t sc = 0;
                if (live && ks < ksteps) {
                    x = *reinterpret_cast<const i32x4 *>(codes + row * (ksteps * 64) + ks * 64 + g * 16);
                    sc = scales[row * (ksteps * 4) + ks * 4 + g];
                }
                *reinterpret_cast<i32x4 *>(t + ks * 1024 + lane * 16) = x;
                packed |= sc << (8 * b);
                float e = 0.0f;
#pragma unroll
                for (int c = 0; c < 4; ++c) {
                    float v[8];
                    mx_decode8<4>(u32x2{(uint32_t)x[c], 0}, v);
#pragma unroll
                    for (int u = 0; u < 8; ++u) e = fmaf(v[u], v[u], e);
                }
                const double f = mx_factor(sc);
                q += (double)e * f * f;
            }
            if (r < (KS + 3) / 4) *reinterpret_cast<uint32_t *>(t + T::SCALES + r * 256 + lane * 4) = packed;
        }
    }
    q += __shfl_xor(q, 16);
    q += __shfl_xor(q, 32);
    if constexpr (WPT > 1) {
        if (g == 0) part[wave][lr] = q;
        __syncthreads();
        q = 0.0;
#pragma unroll
        for (int w = 0; w < WPT; ++w) q += part[wave / WPT * WPT + w][lr];
    }
    if (there && turn == 0 && g == 0) *reinterpret_cast<float *>(t + T::BIAS + lr * 4) = live ? (float)(-0.5 * q) : -FLT_MAX;
}

// Tiles (group, member) in memory; slots behind the last member are left alone.
constexpr int mx_pack_waves(int ks) { return ks <= 4 ? 1 : ks <= 8 ? 2 : 4; }

template <int KS>
__global__ __launch_bounds__(256) void mx_sets_pack_kernel(const uint8_t *__restrict__ codes,
                                                           const uint8_t *__restrict__ scales, int64_t n, int ksteps,
                                                           const int32_t *__restrict__ sets, int64_t l, int k,
                                                           int64_t ntiles, uint8_t *__restrict__ tiles) {
    constexpr int WPT = mx_pack_waves(KS), TILES = 4 / WPT;
    __shared__ double part[4][16];
    const int64_t i = flat_block() * TILES + (threadIdx.x >> 6) / WPT;
    const int slots = (k + 1) / 2 * 2;
    const int64_t grp = i / slots;
    const int p = (int)(i - grp * slots);
    mx_pack_tile<KS, WPT>(codes, scales, n, ksteps, sets, l, k, grp, p, i < ntiles && p < k,
                          tiles + i * MxTile<KS>::BYTES, part);
}

// GATHER: the workgroup makes its tiles itself, all of them at once in LDS (they
// fit), from the sets.
template <int KS, int RT, int WAVES, bool GATHER>
__global__ __launch_bounds__(WAVES * 64, 2) void mx_sets_kernel(const uint8_t *__restrict__ codes,
                                                                const uint8_t *__restrict__ scales, int64_t n, int ksteps,
                                                                const uint8_t *__restrict__ tiles,
                                                                const int32_t *__restrict__ sets, int64_t l, int members,
                                                                int ngroups, int gpc, int nrb,
                                                                float *__restrict__ partials, int64_t lpad) {
    using P = MxSetsPlan<KS, RT, WAVES>;
    using T = MxTile<KS>;
    const int64_t parts = (n + kMxSetRows - 1) / kMxSetRows;
    constexpr int SR = (KS + 3) / 4;  // scale registers of a row tile
    extern __shared__ __align__(16) unsigned char smem[];
    const int tid = threadIdx.x, lane = tid & 63, lr = lane & 15, g = lane >> 4;
    const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int64_t b = flat_block(), chunk = b / nrb;
    const int rb = (int)(b - chunk * nrb);
    const int64_t g0 = chunk * gpc;
    if (g0 >= ngroups) return;
    const int groups = (int)min((int64_t)gpc, ngroups - g0), pairs = (members + 1) / 2, units = groups * pairs;

    const uint8_t *stream = tiles + g0 * pairs * (int64_t)P::UNIT;
    const int stages = GATHER ? 1 : (units + P::UPS - 1) / P::UPS, ups = GATHER ? units : P::UPS;
    auto issue = [&](int st) {
        const int64_t at = (int64_t)st * P::STAGE, left = (int64_t)units * P::UNIT - at;
        const auto win = window_rsrc(stream + at, (uint32_t)max((int64_t)0, min((int64_t)P::STAGE, left)));
        unsigned char *buf = smem + st % P::DEPTH * P::BUF;
#pragma unroll
        for (int i = 0; i < P::LOADS; ++i)
            window_to_lds16(win, buf + (i * P::THREADS + wave * 64) * 16, (uint32_t)((i * P::THREADS + tid) * 16));
    };
    if constexpr (GATHER) {
        for (int i = wave; i < 2 * units; i += WAVES) {
            const int q = i / (2 * pairs), p = i - q * 2 * pairs;
            mx_pack_tile<KS, 1>(codes, scales, n, ksteps, sets, l, members, g0 + q, p, p < members, smem + i * T::BYTES, nullptr);
        }
    } else {
#pragma unroll
        for (int st = 0; st < P::DEPTH - 1; ++st) issue(st);
    }

    // The points, and their scales as the tiles have theirs.
    const int row_bytes = ksteps * 64, row_scales = ksteps * 4;
    const int64_t row0 = (int64_t)rb * P::ROWS, rows = min((int64_t)P::ROWS, n - row0);
    const auto vwin = window_rsrc(codes + row0 * row_bytes, (uint32_t)(rows * row_bytes));
    const auto swin = window_rsrc(scales + row0 * row_scales, (uint32_t)(rows * row_scales));
    i32x4 a[RT][KS];
    int as[RT][SR];
#pragma unroll
    for (int rt = 0; rt < RT; ++rt) {
        const int row = (wave * RT + rt) * 16 + lr;
        uint32_t w[KS];
#pragma unroll
        for (int ks = 0; ks < KS; ++ks) {
            a[rt][ks] = window_load16<i32x4>(vwin, ks < ksteps ? (uint32_t)(row * row_bytes + ks * 64 + g * 16) : kDeadOffset);
            w[ks] = __float_as_uint(window_load4(swin, ks < ksteps ? (uint32_t)(row * row_scales + ks * 4) : kDeadOffset));
        }
#pragma unroll
        for (int q = 0; q < SR; ++q) as[rt][q] = 0;
#pragma unroll
        for (int ks = 0; ks < KS; ++ks) as[rt][ks / 4] |= (int)((w[ks] >> (8 * g) & 255u) << (8 * (ks % 4)));
    }

    f32x4 m[RT];
#pragma unroll
    for (int rt = 0; rt < RT; ++rt) m[rt] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};  // e0

    auto tile = [&](const unsigned char *t, f32x4(&acc)[RT]) {
        const float bias = *reinterpret_cast<const float *>(t + T::BIAS + lr * 4);
        int bs[SR];
#pragma unroll
        for (int q = 0; q < SR; ++q) bs[q] = *reinterpret_cast<const int *>(t + T::SCALES + q * 256 + lane * 4);
#pragma unroll
        for (int rt = 0; rt < RT; ++rt) acc[rt] = f32x4{bias, bias, bias, bias};
        auto step = [&](auto kc) {
            constexpr int ks = decltype(kc)::value;
            const i32x4 x = *reinterpret_cast<const i32x4 *>(t + ks * 1024 + lane * 16);
#pragma unroll
            for (int rt = 0; rt < RT; ++rt)
                acc[rt] = mx_mma<ks % 4, ks % 4>(a[rt][ks], x, acc[rt], as[rt][ks / 4], bs[ks / 4]);
        };
        each_step(step, std::make_integer_sequence<int, KS>{});
    };

    int q = 0;
    int64_t grp = g0;
    // The end of a set group: its sums, and the maximum back to e0's.
    auto finish = [&] {
#pragma unroll
        for (int i = 0; i < RT / 2; ++i) {
            const f32x4 u = m[2 * i] + m[2 * i + 1];
            float s = (u[0] + u[2]) + (u[1] + u[3]);
            s += __shfl_xor(s, 16);
            s += __shfl_xor(s, 32);
            const int64_t part = (row0 + wave * RT * 16) / kMxSetRows + i;
            if (g == 0 && part < parts) partials[part * lpad + grp * 16 + lr] = s;
            m[2 * i] = m[2 * i + 1] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
        }
        q = 0;
        ++grp;
    };
    if constexpr (P::AHEAD && !GATHER) {
        i32x4 b[KS];
        int bs[SR];
        float bias;
        auto read = [&](const unsigned char *t, int ks) {
            b[ks] = *reinterpret_cast<const i32x4 *>(t + ks * 1024 + lane * 16);
            if (ks % 4 == 3 || ks == KS - 1) bs[ks / 4] = *reinterpret_cast<const int *>(t + T::SCALES + ks / 4 * 256 + lane * 4);
        };
        auto read_bias = [&](const unsigned char *t) { bias = *reinterpret_cast<const float *>(t + T::BIAS + lr * 4); };
        // The tile at hand, and the next one's operands over those just used.
        auto tile_then = [&](const unsigned char *next, f32x4(&acc)[RT]) {
            __builtin_amdgcn_sched_barrier(0);
#pragma unroll
            for (int rt = 0; rt < RT; ++rt) acc[rt] = f32x4{bias, bias, bias, bias};
            read_bias(next);
            auto step = [&](auto kc) {
                constexpr int ks = decltype(kc)::value;
#pragma unroll
                for (int rt = 0; rt < RT; ++rt)
                    acc[rt] = mx_mma<ks % 4, ks % 4>(a[rt][ks], b[ks], acc[rt], as[rt][ks / 4], bs[ks / 4]);
                read(next, ks);
                __builtin_amdgcn_sched_barrier(0);
            };
            each_step(step, std::make_integer_sequence<int, KS>{});
        };
        asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
        __syncthreads();
        read_bias(smem);
#pragma unroll
        for (int ks = 0; ks < KS; ++ks) read(smem, ks);
        for (int st = 0; st < stages; ++st) {
            asm volatile("s_waitcnt vmcnt(%0)" ::"n"((P::DEPTH - 3) * P::LOADS) : "memory");  // stage st + 1
            __syncthreads();
            issue(st + P::DEPTH - 1);
            const unsigned char *buf = smem + st % P::DEPTH * P::BUF, *next_buf = smem + (st + 1) % P::DEPTH * P::BUF;
            const int last = min(ups, units - st * ups);
            for (int u = 0; u < last; ++u) {
                const unsigned char *t = buf + u * P::UNIT, *next = u + 1 < last ? t + P::UNIT : next_buf;
                f32x4 x[RT], y[RT];
                const bool two = 2 * q + 1 < members;
                tile_then(two ? t + T::BYTES : next, x);
                if (two) {
                    tile_then(next, y);
#pragma unroll
                    for (int rt = 0; rt < RT; ++rt)
#pragma unroll
                        for (int i = 0; i < 4; ++i) m[rt][i] = fmaxf(fmaxf(m[rt][i], x[rt][i]), y[rt][i]);
                } else {
#pragma unroll
                    for (int rt = 0; rt < RT; ++rt)
#pragma unroll
                        for (int i = 0; i < 4; ++i) m[rt][i] = fmaxf(m[rt][i], x[rt][i]);
                }
                if (++q == pairs) finish();
            }
        }
        asm volatile("s_waitcnt vmcnt(0)" ::: "memory");  // the last copies
        return;
    }
    for (int st = 0; st < stages; ++st) {
        if constexpr (!GATHER) asm volatile("s_waitcnt vmcnt(%0)" ::"n"(P::LOADS) : "memory");
        __syncthreads();
        if constexpr (!GATHER) issue(st + 2);
        const unsigned char *buf = smem + st % 3 * P::BUF;
        const int last = min(ups, units - st * ups);
        for (int u = 0; u < last; ++u) {
            const unsigned char *t = buf + u * P::UNIT;
            f32x4 x[RT], y[RT];
            tile(t, x);
            if (2 * q + 1 < members) {
                tile(t + T::BYTES, y);
#pragma unroll
                for (int rt = 0; rt < RT; ++rt)
#pragma unroll
                    for (int i = 0; i < 4; ++i) m[rt][i] = fmaxf(fmaxf(m[rt][i], x[rt][i]), y[rt][i]);
            } else {
#pragma unroll
                for (int rt = 0; rt < RT; ++rt)
#pragma unroll
                    for (int i = 0; i < 4; ++i) m[rt][i] = fmaxf(m[rt][i], x[rt][i]);
            }
            if (++q == pairs) finish();
        }
    }
    asm volatile("s_waitcnt vmcnt(0)" ::: "memory");  // the last copies
}

// How a launch splits its work: set groups per workgroup, chosen by rounds of
// workgroups over the CUs, times the instructions of the groups a CU works on
// and what a workgroup starts with (the first stages and its points).  Two row
// tiles leave LDS reads about as long as the instructions, and one wavefront to
// a SIMD little to cover them.
template <int KS, int RT, int WAVES>
double mx_sets_cost(const MxSetsArgs &x, int64_t groups, int64_t *gpc) {
    using P = MxSetsPlan<KS, RT, WAVES>;
    const int64_t nrb = (x.n + P::ROWS - 1) / P::ROWS, cus = std::max<int64_t>(1, device_cu_count());
    const int64_t resident = std::min(WAVES > 4 ? 1 : RT > 2 ? 2 : 4, kLdsBytes / P::LDS);
    const double stall = RT > 2 ? 1.0 : P::AHEAD ? 1.35 : resident * WAVES > 4 ? 1.5 : 1.9;
    const double group = (double)x.k * KS * RT * 16.0 * (WAVES / 4) * stall, start = 4000.0 + 500.0 * KS;
    const int64_t most = std::min(groups, std::max<int64_t>(1, kMxMembers / ((x.k + 1) / 2)));
    double best = 0.0;
    for (int64_t c = 1; c <= most; c = c < 16 ? c + 1 : c + c / 8) {
        const int64_t wgs = nrb * ((groups + c - 1) / c), each = std::min(resident, (wgs + cus - 1) / cus);
        const int64_t rounds = (wgs + cus * resident - 1) / (cus * resident);
        const double cost = (double)rounds * ((double)(c * each) * group + start);
        if (c == 1 || cost < best) best = cost, *gpc = c;
    }
    return best;
}

template <int KS, int RT, int WAVES, bool GATHER = false>
hipError_t mx_sets_launch(const MxSetsArgs &x, int64_t groups, int64_t gpc, hipStream_t st) {
    using P = MxSetsPlan<KS, RT, WAVES>;
    auto kern = mx_sets_kernel<KS, RT, WAVES, GATHER>;
    static std::atomic<bool> ready[kMaxDevices];  // the attribute holds for one device
    const int dev = current_device();
    if (dev < 0) return hipErrorInvalidDevice;
    if (!ready[dev].load(std::memory_order_acquire)) {
        const hipError_t e = hipFuncSetAttribute((const void *)kern, hipFuncAttributeMaxDynamicSharedMemorySize, P::LDS);
        if (e != hipSuccess) return e;
        ready[dev].store(true, std::memory_order_release);
    }
    const int64_t nrb = (x.n + P::ROWS - 1) / P::ROWS;
    hipLaunchKernelGGL(kern, flat_grid(nrb * ((groups + gpc - 1) / gpc), P::THREADS), dim3(P::THREADS), P::LDS, st, x.codes,
                       x.scales, x.n, (int)(mx_padded(x.d) / kMxRow), x.work, x.sets, x.l, (int)x.k, (int)groups, (int)gpc,
                       (int)nrb, x.partials, x.lpad);
    return hipGetLastError();
}

// Tiles, then the sums: wavefronts with RT row tiles where the points fill the
// chip that way, workgroups of four with two where they do not.
template <int KS, int RT, int WAVES>
hipError_t mx_sets_run(const MxSetsArgs &x, hipStream_t st) {
    const int64_t groups = x.lpad / 16, slots = (x.k + 1) / 2 * 2, ntiles = groups * slots;
    if (x.k > kMxMembers || groups > INT32_MAX) return hipErrorInvalidValue;
    int64_t gpc = 1, gpc2 = 1;
    const bool large = mx_sets_cost<KS, RT, WAVES>(x, groups, &gpc) <= mx_sets_cost<KS, 2, 4>(x, groups, &gpc2);
    // Few short tiles: each workgroup makes its own, which saves the launch that
    // stages them (10 000 x 64, 48 sets of 8: 13.3 -> 10.2 us a call).
    if constexpr (KS <= 2) {
        using P = MxSetsPlan<KS, 2, 4>;
        const int64_t units = gpc2 * slots / 2;
        if (!large && units <= kMxGatherUnits && units * P::UNIT <= P::LDS)
            return mx_sets_launch<KS, 2, 4, true>(x, groups, gpc2, st);
    }
    hipLaunchKernelGGL(mx_sets_pack_kernel<KS>, flat_grid((ntiles * mx_pack_waves(KS) + 3) / 4, 256), dim3(256), 0, st, x.codes,
                       x.scales, x.n, (int)(mx_padded(x.d) / kMxRow), x.sets, x.l, (int)x.k, ntiles, x.work);
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
    if (large) return mx_sets_launch<KS, RT, WAVES>(x, groups, gpc, st);
    return mx_sets_launch<KS, 2, 4>(x, groups, gpc2, st);
}

}  // namespace exemcl
