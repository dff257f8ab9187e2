// What the files that hold C entry points share on the host.
#pragma once

#include <hip/hip_runtime.h>
#include <stddef.h>

#include "../../include/moe.h"

namespace moe {

// records the text that moe_last_error returns on this thread; returns st
moe_status fail(moe_status st, const char* fmt, ...);

inline size_t align_up(size_t v, size_t a) { return (v + a - 1) / a * a; }

}  // namespace moe

#define HIP_TRY(expr)                                                                   \
  do {                                                                                  \
    hipError_t e_ = (expr);                                                             \
    if (e_ != hipSuccess) return moe::fail(MOE_ERR_HIP, "%s: %s", #expr, hipGetErrorString(e_)); \
  } while (0)
