// What the files of the C ABI share: the failure of an entry point and its message.
#pragma once
#include "samp_common.h"

#include <stddef.h>

namespace samp {

// keeps the message for samp_last_error() of this thread and returns `code`
int fail(int code, const char *fmt, ...) __attribute__((format(printf, 2, 3)));

inline bool aligned(const void *p, size_t a) { return (reinterpret_cast<uintptr_t>(p) % a) == 0; }

}  // namespace samp

#define HIP_TRY(expr)                                                                               \
    do {                                                                                            \
        hipError_t e_ = (expr);                                                                     \
        if (e_ != hipSuccess) return fail(SAMP_ERR_HIP, "%s: %s", #expr, hipGetErrorString(e_));    \
    } while (0)
