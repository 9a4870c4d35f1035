// cf_wgrad_f16.hip -- the weight gradient (cf_wgrad.h) in fp16.
#include "cf_wgrad.h"

namespace cf {

hipError_t launch_wgrad_f16(const WGradArgs &a, int tile, hipStream_t st) { return launch_type<F16, false>(a, tile, st); }

}  // namespace cf
