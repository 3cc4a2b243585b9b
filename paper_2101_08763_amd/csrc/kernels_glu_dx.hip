// kernels_glu_dx.hip -- dx = dg Wg + du Wu: one sum over both, rounded once.
#include "glu_tile.hpp"

namespace exemcl {

hipError_t launch_glu_dx(int prec, const DenseArgs &a, hipStream_t st) {
    DenseLaunch l = dense_args(a);
    l.matrices = 2;
    if (prec == P_FP32) return dense_run<float, ALONG, ACROSS, STORE>(l, st);
    if (prec == P_FP16) return dense_run<_Float16, ALONG, ACROSS, STORE>(l, st);
    return dense_run<__bf16, ALONG, ACROSS, STORE>(l, st);
}

int64_t glu_dx_partial(int prec, int64_t M, int64_t N, int64_t K) {
    return prec == P_FP32 ? dense_partial_bytes<float>(M, N, K, 1, 2) : dense_partial_bytes<_Float16>(M, N, K, 1, 2);
}

}  // namespace exemcl
