// The calling thread's last error message, shared by every C entry point.
#pragma once

#include <hip/hip_runtime.h>

#include "../../include/libmalt.h"

namespace malt {

// Records the message malt_last_error() returns and hands back `st`.
malt_status_t fail(malt_status_t st, const char* fmt, ...) __attribute__((format(printf, 2, 3)));
malt_status_t hip_fail(hipError_t e, const char* what);

}  // namespace malt
