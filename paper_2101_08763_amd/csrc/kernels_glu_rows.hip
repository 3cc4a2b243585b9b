// kernels_glu_rows.hip -- the gated block on few rows, weights of the rows' type.
#include <algorithm>
#include <cmath>

#include "glu_rows.hpp"

namespace exemcl {

namespace {

// 16 MT rows to a workgroup: more rows share a weight, and fewer workgroups share
// the CUs.  Time of a launch: a wavefront's blocks of 128 coordinates, at so many
// us by type and MT; where the workgroups take turns on a CU those of all, and
// something for each; or the weights from memory.  Estimate and measured (us, MT =
// 1, 2, 4):
//   bf16  16 x 4096 x 8192   32 / 34 / 49    31 / 32 / 38
//         32 x 4096 x 8192   48 / 34 / 49    47 / 37 / 41
//         64 x 1024 x 2048   10 / 8 / 10     8.7 / 8.5 / 10.4
//         64 x 8192 x 512    25 / 33 / 47    24 / 31 / 45
//   fp32  16 x 4096 x 4096   28 / 39 / 58    30 / 41 / 53
//         64 x 1024 x 2048   18 / 14 / 18    17 / 12 / 17
//         128 x 4096 x 4096  195 / 144 / 111 191 / 135 / 102
//         333 x 301 x 1111   25 / 21 / 16    21 / 15 / 15
// Rows that begin at odd multiples of 2 bytes load at 2/5 of the rate (bf16 64 x 1001 x
// 3000 17, 64 x 1000 x 3000 10).
// Tiles of the dense kernels (glu_tile.hpp) take 41 us for 32 x 4096 x 8192 and 40
// for 100 of bf16 (rows: 37 and 90), 219 for 128 x 4096 x 4096 of fp32 and 24 for
// 333 x 301 x 1111 (rows: 15).
struct Choice {
    int mt;
    double us;
};
Choice choose(int prec, int64_t n, int64_t d, int64_t f) {
    const bool wide = prec == P_FP32;
    constexpr double kBlock[2][3] = {{2.6, 3.6, 5.4}, {5.6, 8.4, 13.0}};
    const double cus = (double)std::max<int64_t>(1, device_cu_count()), blocks = (double)w4_blocks(d);
    // The longest share of a wavefront: blocks, or steps of 32 where blocks are few.
    const double longest = d / kW4Block < kRowsWaves ? std::ceil((double)((d + 31) / 32) / kRowsWaves) / 4.0 : std::ceil(blocks / kRowsWaves);
    const double odd = !wide && d % 2 ? 2.5 : 1.0;
    const double bytes = (double)f * (double)d * (wide ? 8.0 : 4.0);
    Choice best{1, 0.0};
    for (int i = 0; i < 3; ++i) {
        const int mt = 1 << i;
        const double workgroups = (double)((f + 15) / 16) * (double)((n + 16 * mt - 1) / (16 * mt)) / cus;
        // (of fp32 one workgroup is on a CU at a time)
        const double rounds = wide && workgroups > 1.0 ? std::ceil(workgroups) : workgroups;
        const double turns = std::max(longest, rounds * blocks / kRowsWaves);
        const double us = std::max(4.0 + turns * kBlock[wide][i] * odd + workgroups * (wide ? 1.5 : 0.5), 3.0 + bytes / 4.6e6);
        if (best.us == 0.0 || us < best.us) best = {mt, us};
    }
    return best;
}

template <typename T>
hipError_t run(int prec, const RowsArgs &r, hipStream_t st) {
    const int mt = choose(prec, r.n, r.d, r.f).mt;
    if (mt == 1) return rows_launch<T, 0, true, 1, 1, 1>(r, st);
    if (mt == 2) return rows_launch<T, 0, true, 1, 2, 1>(r, st);
    return rows_launch<T, 0, true, 1, 4, 1>(r, st);
}

}  // namespace

bool glu_takes_rows(int prec, int64_t n, int64_t d, int64_t f, bool staged) {
    if (n <= 64 && staged) return true;  // which takes no temporary memory
    return choose(prec, n, d, f).us <= glu_tiles_us(prec, n, d, f, staged);
}

hipError_t launch_glu_rows(int prec, const GluArgs &a, hipStream_t st) {
    const RowsArgs r{a.x, a.n, a.d, {a.wg, a.wu}, {nullptr, nullptr}, a.f, {a.bg, a.bu}, a.act, a.h, a.g, a.u, 0, 0};
    if (prec == P_FP32) return run<float>(prec, r, st);
    if (prec == P_FP16) return run<_Float16>(prec, r, st);
    return run<__bf16>(prec, r, st);
}

}  // namespace exemcl
