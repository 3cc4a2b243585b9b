// kernels_mx_sets_short.hip -- sets on 4-bit rows of up to 768 coordinates.
#include "mx_sets.hpp"

namespace exemcl {

hipError_t mx_sets_short(int ks, const MxSetsArgs &x, hipStream_t st) {
    switch (ks) {
    case 1: return mx_sets_run<1, 8, 4>(x, st);
    case 2: return mx_sets_run<2, 8, 4>(x, st);
    case 3: return mx_sets_run<3, 8, 4>(x, st);
    case 4: return mx_sets_run<4, 8, 4>(x, st);
    case 5: return mx_sets_run<5, 4, 4>(x, st);
    default: return mx_sets_run<6, 4, 4>(x, st);
    }
}

}  // namespace exemcl
