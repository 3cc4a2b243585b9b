// kernels_glu_forward.hip -- the gated block on many rows: x and both weights lie
// along the contraction.
#include "glu_tile.hpp"

namespace exemcl {

hipError_t launch_glu_forward(int prec, const DenseArgs &a, hipStream_t st) {
    const DenseLaunch l = dense_args(a);
    if (prec == P_FP32) return dense_run<float, ALONG, ALONG, GLU>(l, st);
    if (prec == P_FP16) return dense_run<_Float16, ALONG, ALONG, GLU>(l, st);
    return dense_run<__bf16, ALONG, ALONG, GLU>(l, st);
}

}  // namespace exemcl
