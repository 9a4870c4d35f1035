// cf_wgrad_norm_f16.hip -- the weight gradient (cf_wgrad.h) in fp16 after a layer norm.
#include "cf_wgrad.h"

namespace cf {

hipError_t launch_wgrad_norm_f16(const WGradArgs &a, int tile, hipStream_t st) { return launch_type<F16, true>(a, tile, st); }

}  // namespace cf
