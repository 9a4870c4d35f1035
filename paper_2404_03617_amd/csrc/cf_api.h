// cf_api.h -- error reporting shared by the files of the C ABI layer.
#pragma once

#include "convfirst.h"

#include <hip/hip_runtime.h>

namespace cf {

// Stores the calling thread's message for cf_last_error and returns s.
cf_status api_fail(cf_status s, const char *fmt, ...) __attribute__((format(printf, 2, 3)));

// The status of a call whose launches returned e; clears the message on success.
cf_status api_done(hipError_t e, const char *what);

}  // namespace cf
