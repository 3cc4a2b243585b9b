// kernels_glu_dw.hip -- dWg = dg' x and dWu = du' x in one launch: the rows are
// what is summed over, and both operands lie across it.
#include "glu_tile.hpp"

namespace exemcl {

hipError_t launch_glu_dw(int prec, const DenseArgs &a, hipStream_t st) {
    DenseLaunch l = dense_args(a);
    l.pairs = a.C && a.C2 ? 2 : 1;
    if (!a.C) l.A = l.A2, l.C = l.C2;
    if (prec == P_FP32) return dense_run<float, ACROSS, ACROSS, STORE>(l, st);
    if (prec == P_FP16) return dense_run<_Float16, ACROSS, ACROSS, STORE>(l, st);
    return dense_run<__bf16, ACROSS, ACROSS, STORE>(l, st);
}

int64_t glu_dw_partial(int prec, int64_t M, int64_t N, int64_t K, int pairs) {
    return prec == P_FP32 ? dense_partial_bytes<float>(M, N, K, pairs, 1) : dense_partial_bytes<_Float16>(M, N, K, pairs, 1);
}

}  // namespace exemcl
