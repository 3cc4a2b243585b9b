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

// One launch more lays the operands out (11 us for 100 x 300 x 500 in bf16, where a
// launch of tiles takes 6); weights come at 3.5 TB/s at most (64 and 128 x 4096 x
// 8192 in bf16: 41 us each).
double glu_tiles_us(int prec, int64_t n, int64_t d, int64_t f, bool staged) {
    const bool wide = prec == P_FP32;
    const double weights = (double)f * (double)d * 2.0, values = weights + (double)n * (double)d;
    const double tiles = dense_choice(n, f, 1, (d + 63) / 64 * (wide ? Operand<float>::PRODUCTS : 1), true, false).us;
    return std::max(tiles, 3.0 + weights * (wide ? 6.0 : 2.0) / 3.5e6) + (staged ? 5.5 + values * (wide ? 10.0 : 4.0) / 5e6 : 0.0);
}

}  // namespace exemcl
