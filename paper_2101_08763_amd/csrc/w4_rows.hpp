// w4_rows.hpp -- products by 4-bit weights and the gated block on them: the sizes'
// kernels (instantiated in kernels_w4_*.hip, one per type of the rows).
#pragma once

#include "w4_tile.hpp"

namespace exemcl {

template <typename T, int GROUP, bool GLU>
hipError_t w4_sized(const RowsArgs &r, hipStream_t st) {
    using P = W4TilePlan<T, GROUP>;
    constexpr bool WIDE = sizeof(T) == 4;
    const int64_t cus = std::max<int64_t>(1, device_cu_count()), mats = GLU ? 2 : 1, pairs = (r.f + 31) / 32;
    // With few rows, 32 of them and two tiles of weights to a workgroup read least; with
    // fewer results 16 rows, or one tile, where two blocks ahead pay (us, 16 rows and one
    // tile / 16 and two / 32 and two, bf16 by groups of 128: 16 x 4096 x 8192 11.2 / 7.9 / -,
    // 16 x 8192 x 4096 10.8 / 11.6 / -, 64 x 4096 x 8192 35 / 21 / 20, 64 x 4096 x 2048
    // 11.2 / 9.1 / 11.4, 64 x 8192 x 1024 11.8 / 12.0 / 19; fp32, two matrices by 64:
    // 32 x 4096 x 8192 48 / 28 / 27).
    auto fills = [&](int64_t n) { return 10 * pairs * ((r.n + n - 1) / n) >= 7 * cus; };
    // The block by groups of 32 spills registers where a workgroup has two tiles (us, one
    // tile / two): fp32 and 16 rows 36 of them, 83 / 133 for 1 x 4096 x 32768, and it takes one;
    // 32 rows 38, 189 / 158 for 17; fp16 and bf16 8 and 19, 52 / 54 for 1, 62 / 58 for 16 and
    // 115 / 103 for 32.
    constexpr bool ONE = WIDE && GLU && GROUP == 32;
    const int xt = r.n > 16 && fills(32) ? 2 : 1, wt = xt == 2 || (!ONE && fills(16)) ? 2 : 1;
    // Those, with the weights read again (from the caches) for every 16 xt rows, or tiles
    // of 128 rows (fp32: 64) through LDS, whichever is estimated to take less.  Few rows:
    // what the launch, the instructions for 16 rows and a workgroup's start and join take;
    // tiles: rounds of workgroups, their blocks of 128 coordinates, start and end.
    // Measured (us, few rows / tiles; bf16 by groups of 128 where nothing else is said):
    //   1 x 4096 x 8192    6.9 / 60     8 x 256 x 8192      3.0 / 8.6  128 x 4096 x 8192  36 / 64
    //   1 x 4096 x 131072  58 / 150     17 x 40 x 700       3.3 / 8.8  256 x 4096 x 8192  68 / 64
    //   16                 79 / 151     1 x 128 x 131072    14 / 13    512 x 4096 x 8192  131 / 66
    //   32                 138 / 155    64 x 256 x 65536    25 / 14    256 x 1536 x 1536, by 64  10 / 34
    //   two matrices 512 x 512 x 2048  18 / 15    fp32 128 x 4096 x 4096  39 / 84
    // Of 2 051 sizes with an even d (1 to 1 000 rows) the choice takes 1.4 % more than the
    // better one on average.  Rows of an odd d load at less than half the rate in both
    // (512 x 1001 x 3000 32 / 32, 1008: 17 / 23), and the choice is as good without a term
    // for them.
    const double rows = 3.8 + (double)((r.n + 15) / 16 * mats) * (double)r.f * (double)r.d * (WIDE ? 2.7e-7 : GROUP == 32 ? 1.7e-7 : 1.2e-7) +
                        1.5 * (double)((r.n + 16 * xt - 1) / (16 * xt) * ((r.f + 16 * wt - 1) / (16 * wt))) / (double)cus;
    const int64_t rounds = ((r.n + P::ROWS - 1) / P::ROWS * ((r.f * mats + 255) / 256) + cus - 1) / cus;
    const double block = WIDE ? 2.9 : GROUP == 128 ? 2.2 : GROUP == 64 ? 2.4 : 3.2;
    if (rows > 3.0 + (double)rounds * ((double)w4_blocks(r.d) * block + 2.5)) return w4_tile_launch<T, GROUP, GLU>(r, st);
    if (xt == 2) return rows_launch<T, GROUP, GLU, 2, 2, 1>(r, st);
    if constexpr (!ONE)
        if (wt == 2) return rows_launch<T, GROUP, GLU, 2, 1, 1>(r, st);
    return rows_launch<T, GROUP, GLU, 1, 1, (GROUP >= 64 ? 2 : 1)>(r, st);
}

template <typename T>
hipError_t w4_typed(const W4Args &a, hipStream_t st) {
    const RowsArgs r{a.x, a.n, a.d, {a.wg, a.wu}, {a.wg_words, a.wu_words}, a.f, {a.bg, a.bu}, a.act, a.y, nullptr, nullptr, 0, 0};
    if (a.group == 32) return a.wu ? w4_sized<T, 32, true>(r, st) : w4_sized<T, 32, false>(r, st);
    if (a.group == 64) return a.wu ? w4_sized<T, 64, true>(r, st) : w4_sized<T, 64, false>(r, st);
    return a.wu ? w4_sized<T, 128, true>(r, st) : w4_sized<T, 128, false>(r, st);
}

hipError_t w4_run_f32(const W4Args &a, hipStream_t st);
hipError_t w4_run_f16(const W4Args &a, hipStream_t st);
hipError_t w4_run_bf16(const W4Args &a, hipStream_t st);

}  // namespace exemcl
