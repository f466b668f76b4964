// Error text of the calling thread, shared by the host files of libsalad.
#pragma once
#include <hip/hip_runtime.h>

#include "../../include/salad.h"

namespace salad {

__attribute__((visibility("hidden"), format(printf, 2, 3))) salad_status fail(salad_status st, const char *fmt, ...);
__attribute__((visibility("hidden"))) salad_status hip_fail(hipError_t e, const char *what);

}  // namespace salad
