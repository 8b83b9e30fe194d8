// The C-ABI layer's errors: both set the calling thread's message
// (splash_last_error) and return the status.
#pragma once

#include <hip/hip_runtime.h>

namespace splash {

int fail(int status, const char* fmt, ...) __attribute__((format(printf, 2, 3)));
int hip_fail(hipError_t e, const char* what);

}  // namespace splash
