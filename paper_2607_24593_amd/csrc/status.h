// Status reporting shared by the C entry points (defined in api.hip).
#pragma once

#include <hip/hip_runtime.h>

#include "pivot.h"

namespace pivot {

// Records the message as the calling thread's last error and returns s.
pivot_status fail(pivot_status s, const char* fmt, ...) __attribute__((format(printf, 2, 3)));
pivot_status hip_check(hipError_t e, const char* what);

}  // namespace pivot
