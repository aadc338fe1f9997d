// What the host sides of the library share: errors (ee_last_error) and checked HIP calls.
#pragma once

#include <hip/hip_runtime.h>

#include "../../include/ee.h"

namespace ee {
int fail(int code, const char *fmt, ...) __attribute__((format(printf, 2, 3)));   // notes the message for ee_last_error and returns `code`
}

#define HIP_TRY(expr)                                                                          \
    do {                                                                                       \
        hipError_t e_ = (expr);                                                                \
        if (e_ != hipSuccess)                                                                  \
            return fail(EE_EDEVICE, "%s failed: %s (%s:%d)", #expr, hipGetErrorString(e_), __FILE__, __LINE__); \
    } while (0)
