// kernels_w4_f16.hip -- 4-bit weights, rows of type _Float16.
#include "w4_rows.hpp"

namespace exemcl {

hipError_t w4_run_f16(const W4Args &a, hipStream_t st) { return w4_typed<_Float16>(a, st); }

}  // namespace exemcl
