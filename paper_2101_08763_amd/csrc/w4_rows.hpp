// w4_rows.hpp -- products by 4-bit weights and the gated block on them: the sizes'
// kernels (instantiated in kernels_w4_*.hip, one per type of the rows).
#pragma once


#include "w4_tile.hpp"

namespace exemcl {

template <typename T, int GROUP, bool GLU>
hipError_t w4_sized(const RowsArgs &r, hipStream_t st) {
    using P = W4TilePlan<T, GROUP>;
    // Rows at a time with the weights read again (from the caches), or tiles of 128 (fp32:
    // 64) through LDS, whichever is estimated to take less (us, with one and the other,
    // bf16 by groups of 128: 128 x 4096 x 8192 35 / 64, 256 70 / 64; two matrices, 512 x 512 x
    // 2048 18 / 15; by groups of 64: 256 x 1536 x 1536 10 / 34; fp32: 128 x 4096 x 4096 39 / 84).
    const int64_t cus = std::max<int64_t>(1, device_cu_count()), mats = GLU ? 2 : 1, pairs = (r.f + 31) / 32;
    const double rows = 4.0 + (double)((r.n + 31) / 32 * mats) * (double)r.f * (double)r.d *
                                  (sizeof(T) == 4 ? 5.6e-7 : GROUP == 32 ? 3.1e-7 : 2.5e-7);
    const int64_t workgroups = (r.n + P::ROWS - 1) / P::ROWS * ((r.f * mats + 255) / 256);
    const double each = sizeof(T) == 4 ? 3.0 : GROUP == 128 ? 2.0 : GROUP == 64 ? 2.6 : 3.2;
    if (rows <= (double)((workgroups + cus - 1) / cus * w4_blocks(r.d)) * each) {
        // 32 rows and two tiles of weights to a workgroup read least; with fewer results
        // 16 rows, or one tile, where two blocks ahead pay (us, 16 rows and one tile / 16
        // and two / 32 and two, bf16 by groups of 128: 16 x 4096 x 8192 11.2 / 7.9 / -,
        // 16 x 8192 x 4096 10.8 / 11.6 / -, 64 x 4096 x 8192 35 / 21 / 20, 64 x 4096 x 2048
        // 11.2 / 9.1 / 11.4, 64 x 8192 x 1024 11.8 / 12.0 / 19; fp32, two matrices by 64:
        // 32 x 4096 x 8192 48 / 28 / 27).
        auto fills = [&](int64_t n) { return 10 * pairs * ((r.n + n - 1) / n) >= 7 * cus; };
        if (r.n > 16 && fills(32)) return rows_launch<T, GROUP, GLU, 2, 2, 1>(r, st);
        if (fills(16)) return rows_launch<T, GROUP, GLU, 2, 1, 1>(r, st);
        return rows_launch<T, GROUP, GLU, 1, 1, (GROUP >= 64 ? 2 : 1)>(r, st);
    }
    return w4_tile_launch<T, GROUP, GLU>(r, st);
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
