// kernels_mx_sets_wide.hip -- sets on 4-bit rows of 769 to 2 048 coordinates.
#include "mx_sets.hpp"

namespace exemcl {

hipError_t mx_sets_wide(int ks, const MxSetsArgs &x, hipStream_t st) {
    switch (ks) {
    case 8: return mx_sets_run<8, 4, 4>(x, st);
    case 10: return mx_sets_run<10, 2, 8>(x, st);
    case 12: return mx_sets_run<12, 2, 8>(x, st);
    case 14: return mx_sets_run<14, 2, 8>(x, st);
    default: return mx_sets_run<16, 2, 8>(x, st);
    }
}

}  // namespace exemcl
