// cf_mm_logits_bf16.hip -- products of cf_mm.h whose results are logits, bf16.
#include "cf_mm_run.h"

namespace cf {
namespace mm {

template <>
hipError_t launch_lse<BF16>(const Args &a, const LseArgs &e, int tile, hipStream_t st) {
    return launch_tile<BF16, KC, KC, Lse>(a, e, tile, st);
}
template <>
hipError_t launch_dz<BF16>(const Args &a, const DzArgs &e, int tile, hipStream_t st) {
    return launch_tile<BF16, KC, KC, Dz>(a, e, tile, st);
}

}  // namespace mm
}  // namespace cf
