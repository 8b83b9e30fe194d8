// The C-ABI layer's errors: both set the calling thread's message
// (splash_last_error) and return the status.
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

#include "splash_attn.h"

namespace splash {

int fail(int status, const char* fmt, ...) __attribute__((format(printf, 2, 3)));
int hip_fail(hipError_t e, const char* what);

// What every MLA call asks of its descriptor (q_chunk: query rows a request).
int validate_mla_desc(const splash_mla_desc* d, int32_t q_chunk);

}  // namespace splash
