// cf_gnorm_bf16.hip -- group norm (cf_gnorm.h) in bf16.
#include "cf_gnorm.h"

namespace cf {
namespace gnorm {

hipError_t forward_bf16(const Args &a, const Plan &p, int64_t N, int act, hipStream_t st) {
    return forward<BF16>(a, p, N, act, st);
}
hipError_t backward_bf16(const Args &a, const Plan &p, int64_t N, int act, hipStream_t st) {
    return backward<BF16>(a, p, N, act, st);
}

}  // namespace gnorm
}  // namespace cf
