// kernels_w4_f32.hip -- 4-bit weights, rows of type float.
#include "w4_rows.hpp"

namespace exemcl {

hipError_t w4_run_f32(const W4Args &a, hipStream_t st) { return w4_typed<float>(a, st); }

}  // namespace exemcl
