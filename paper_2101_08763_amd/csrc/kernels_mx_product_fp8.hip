// kernels_mx_product_fp8.hip -- products of 8-bit with 4-bit rows.
#include "mx_product.hpp"

namespace exemcl {

hipError_t mx_product_fp8(int prec, const MxProductArgs &a, hipStream_t st) { return product_typed<8>(prec, a, st); }

}  // namespace exemcl
