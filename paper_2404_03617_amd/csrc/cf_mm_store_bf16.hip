// cf_mm_store_bf16.hip -- products of cf_mm.h that are stored as they are, bf16.
#include "cf_mm_run.h"

namespace cf {
namespace mm {

template <>
hipError_t launch_store<BF16, KC, KC>(const Args &a, const StoreArgs &e, int tile, hipStream_t st) {
    return launch_tile<BF16, KC, KC, Store>(a, e, tile, st);
}
template <>
hipError_t launch_store<BF16, KC, RC>(const Args &a, const StoreArgs &e, int tile, hipStream_t st) {
    return launch_tile<BF16, KC, RC, Store>(a, e, tile, st);
}
template <>
hipError_t launch_store<BF16, RC, RC>(const Args &a, const StoreArgs &e, int tile, hipStream_t st) {
    return launch_tile<BF16, RC, RC, Store>(a, e, tile, st);
}

}  // namespace mm
}  // namespace cf
