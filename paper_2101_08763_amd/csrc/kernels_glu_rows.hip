// kernels_glu_rows.hip -- the gated block on few rows, weights of the rows' type.
#include "glu_rows.hpp"

namespace exemcl {

namespace {

template <typename T>
hipError_t run(const RowsArgs &r, hipStream_t st) {
    if (r.n <= 16) return rows_launch<T, 0, true, 1, 1, 1>(r, st);
    if (r.n <= 32) return rows_launch<T, 0, true, 1, 2, 1>(r, st);
    return rows_launch<T, 0, true, 1, 4, 1>(r, st);
}

}  // namespace

bool glu_takes_rows(int, int64_t n, int64_t, int64_t) { return n <= 64; }

hipError_t launch_glu_rows(int prec, const GluArgs &a, hipStream_t st) {
    const RowsArgs r{a.x, a.n, a.d, {a.wg, a.wu}, {nullptr, nullptr}, a.f, {a.bg, a.bu}, a.act, a.h, a.g, a.u, 0, 0};
    if (prec == P_FP32) return run<float>(r, st);
    if (prec == P_FP16) return run<_Float16>(r, st);
    return run<__bf16>(r, st);
}

}  // namespace exemcl
