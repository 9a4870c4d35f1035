// cf_mm_gated_bf16.hip -- the gated feed-forward block's products (cf_mm.h), bf16.
#include "cf_mm_run.h"

namespace cf {
namespace mm {

template <>
hipError_t launch_gated<BF16>(const Args &a, const GatedArgs &e, int tile, hipStream_t st) {
    return launch_tile<BF16, KC, KC, Gated>(a, e, tile, st);
}
template <>
hipError_t launch_gated_back<BF16>(const Args &a, const GatedBackArgs &e, int tile, hipStream_t st) {
    return launch_tile<BF16, KC, RC, GatedBack>(a, e, tile, st);
}

}  // namespace mm
}  // namespace cf
