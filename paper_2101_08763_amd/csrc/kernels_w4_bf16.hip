// kernels_w4_bf16.hip -- 4-bit weights, rows of type __bf16.
#include "w4_rows.hpp"

namespace exemcl {

hipError_t w4_run_bf16(const W4Args &a, hipStream_t st) { return w4_typed<__bf16>(a, st); }

}  // namespace exemcl
