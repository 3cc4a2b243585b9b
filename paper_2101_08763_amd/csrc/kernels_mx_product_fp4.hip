// kernels_mx_product_fp4.hip -- products of 4-bit with 4-bit rows.
#include "mx_product.hpp"

namespace exemcl {

hipError_t mx_product_fp4(int prec, const MxProductArgs &a, hipStream_t st) { return product_typed<4>(prec, a, st); }

}  // namespace exemcl
