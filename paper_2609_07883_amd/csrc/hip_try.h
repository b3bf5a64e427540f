// Turns a failed HIP runtime call into the library's error (internal).
#pragma once

#include <hip/hip_runtime.h>

#include "common.h"

#define HIP_TRY(expr)                                                                           \
    do {                                                                                        \
        hipError_t e_ = (expr);                                                                 \
        if (e_ != hipSuccess) return slw::fail(SLW_EHIP, "%s: %s", #expr, hipGetErrorString(e_)); \
    } while (0)
