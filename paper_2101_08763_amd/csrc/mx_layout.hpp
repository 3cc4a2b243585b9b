// mx_layout.hpp -- how microscaled rows are stored (exemcl.h has the formats).
// A row of d coordinates is padded to whole groups of 128, what one
// matrix-core instruction covers, so every lane vector of 16 code bytes is
// aligned and inside its row.
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

namespace exemcl {

constexpr int kMxBlock = 32, kMxRow = 128;
constexpr int64_t kMxMaxD = int64_t(1) << 22;    // 256 rows within 31-bit byte offsets
constexpr int64_t kMaxNormD = int64_t(1) << 24;
constexpr int kMxSets = 16;                      // sets in a group

enum MxFormat { MX_NONE = 0, MX_FP4 = 4, MX_FP8 = 8 };

__host__ __device__ constexpr int64_t mx_padded(int64_t d) { return (d + kMxRow - 1) / kMxRow * kMxRow; }
__host__ __device__ constexpr int64_t mx_row_bytes(int64_t d, int bits) { return mx_padded(d) * bits / 8; }
__host__ __device__ constexpr int64_t mx_row_scales(int64_t d) { return mx_padded(d) / kMxBlock; }

}  // namespace exemcl
