// w4_rows.hpp -- products by 4-bit weights and the gated block on them: the sizes'
// kernels (instantiated in kernels_w4_*.hip, one per type of the rows).
#pragma once

#include <cmath>

#include "w4_tile.hpp"

namespace exemcl {

template <typename T, int GROUP, bool GLU>
hipError_t w4_sized(const RowsArgs &r, hipStream_t st) {
    // Two blocks ahead pay where a block is few registers (us, one row, bf16, 1 / 2 / 4
    // ahead: 8192 x 4096 by groups of 128 8.8 / 7.8 / 8.2, 1536 x 8192 by 32 4.6 / 5.0 /
    // 8.0); 16 wavefronts to a workgroup spill.
    if (r.n <= 16) return rows_launch<T, GROUP, GLU, 1, 1, (GROUP >= 64 ? 2 : 1)>(r, st);
    if (r.n <= 32) return rows_launch<T, GROUP, GLU, 1, 2, 1>(r, st);
    // Many rows: 64 at a time with the weights read again (from the caches), or tiles of
    // 128 (fp32: 64) through LDS, whichever is estimated to take less (us, with one and
    // the other, bf16 by groups of 128: 128 x 4096 x 8192 38 / 63, 256 73 / 64, 512 142 / 66;
    // by 64: 256 x 1536 x 1536 10 / 34, 1000 28 / 35; fp32: 256 x 4096 x 4096 101 / 99).
    using P = W4TilePlan<T, GROUP>;
    const double mats = GLU ? 2.0 : 1.0, cus = (double)std::max<int64_t>(1, device_cu_count());
    const double rows = (double)((r.n + 63) / 64) * (double)r.f * (double)r.d * mats * (sizeof(T) == 4 ? 1.45e-6 : 6e-7);
    const double workgroups = (double)((r.n + P::ROWS - 1) / P::ROWS) * (double)((r.f * (GLU ? 2 : 1) + 255) / 256);
    const double each = sizeof(T) == 4 ? 3.0 : GROUP == 128 ? 2.0 : GROUP == 64 ? 2.6 : 3.2;
    if (rows <= std::ceil(workgroups / cus) * (double)w4_blocks(r.d) * each)
        return rows_launch<T, GROUP, GLU, GLU ? 1 : 2, 4, 1>(r, st);
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
