// cf_wgrad_bf16.hip -- the weight gradient (cf_wgrad.h) in bf16.
#include "cf_wgrad.h"

namespace cf {

hipError_t launch_wgrad_bf16(const WGradArgs &a, int tile, hipStream_t st) { return launch_type<BF16, false>(a, tile, st); }

}  // namespace cf
