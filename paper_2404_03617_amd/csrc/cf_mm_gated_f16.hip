// cf_mm_gated_f16.hip -- the gated feed-forward block's products (cf_mm.h), fp16.
#include "cf_mm_run.h"

namespace cf {
namespace mm {

template <>
hipError_t launch_gated<F16>(const Args &a, const GatedArgs &e, int tile, hipStream_t st) {
    return launch_tile<F16, KC, KC, Gated>(a, e, tile, st);
}
template <>
hipError_t launch_gated_back<F16>(const Args &a, const GatedBackArgs &e, int tile, hipStream_t st) {
    return launch_tile<F16, KC, RC, GatedBack>(a, e, tile, st);
}

}  // namespace mm
}  // namespace cf
