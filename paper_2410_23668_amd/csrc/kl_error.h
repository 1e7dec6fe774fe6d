// The error message of the calling thread's last failing call, and how entry
// points report one.
#pragma once

#include <string>

#include "kl.h"

namespace kl {

extern thread_local std::string g_last_error;   // kl_last_error()

// Sets the message and returns s.
kl_status fail(kl_status s, const char *fmt, ...) __attribute__((format(printf, 2, 3)));

}  // namespace kl

#define HIP_TRY(expr)                                                                      \
    do {                                                                                   \
        hipError_t e_ = (expr);                                                            \
        if (e_ != hipSuccess)                                                              \
            return fail(e_ == hipErrorOutOfMemory ? KL_ERR_OUT_OF_MEMORY : KL_ERR_HIP,     \
                        "%s failed: %s", #expr, hipGetErrorString(e_));                    \
    } while (0)
