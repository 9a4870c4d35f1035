// cf_gnorm_f16.hip -- group norm (cf_gnorm.h) in fp16.
#include "cf_gnorm.h"

namespace cf {
namespace gnorm {

hipError_t forward_f16(const Args &a, const Plan &p, int64_t N, int act, hipStream_t st) {
    return forward<F16>(a, p, N, act, st);
}
hipError_t backward_f16(const Args &a, const Plan &p, int64_t N, int act, hipStream_t st) {
    return backward<F16>(a, p, N, act, st);
}

}  // namespace gnorm
}  // namespace cf
