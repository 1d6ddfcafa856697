// What the C entry points share on the host: the thread's error text.
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

#include "../../include/treespark.h"

namespace ts {

// Sets the calling thread's error text (ts_last_error) and returns code.
int32_t fail(int32_t code, const char* fmt, ...) __attribute__((format(printf, 2, 3)));
// Clears it, at the start of an entry point.
void clear_error();

#define TS_HIP(call)                                                                     \
  do {                                                                                   \
    hipError_t e_ = (call);                                                              \
    if (e_ != hipSuccess) return fail(TS_EHIP, "%s: %s", #call, hipGetErrorString(e_));  \
  } while (0)

}  // namespace ts
