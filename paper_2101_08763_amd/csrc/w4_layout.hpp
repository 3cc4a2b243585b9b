// w4_layout.hpp -- how weights of 4 bits with group scales are stored (exemcl.h
// has the format): tiles of 16 rows x 128 coordinates, 1 KiB each, in the order in
// which a wavefront's lanes hold the first operand of 16x16x32 instructions, so
// that one load of 16 bytes a lane feeds four of them.
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

namespace exemcl {

constexpr int kW4Rows = 16, kW4Block = 128, kW4Tile = kW4Rows * kW4Block / 2;
constexpr int64_t kW4MaxD = int64_t(1) << 22;

__host__ __device__ constexpr int64_t w4_tiles(int64_t n) { return (n + kW4Rows - 1) / kW4Rows; }
__host__ __device__ constexpr int64_t w4_blocks(int64_t d) { return (d + kW4Block - 1) / kW4Block; }
__host__ __device__ constexpr int64_t w4_groups(int64_t d, int group) { return w4_blocks(d) * (kW4Block / group); }

}  // namespace exemcl
