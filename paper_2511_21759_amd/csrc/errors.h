// Error reporting of the C entry points.
#pragma once
#include <hip/hip_runtime.h>

#include "../../include/odb.h"

namespace odb {

// keeps the message for odb_last_error() on this thread and returns `code`
int fail(int code, const char *fmt, ...);

#define HIP_TRY(expr)                                                                         \
    do {                                                                                      \
        hipError_t e_ = (expr);                                                               \
        if (e_ != hipSuccess) return fail(ODB_E_HIP, "%s: %s", #expr, hipGetErrorString(e_)); \
    } while (0)

}  // namespace odb
