// abi_status.hpp -- what the extern "C" entry points share: the calling
// thread's error message and the checks that fill it.
#pragma once

#include <hip/hip_runtime.h>
#include <stdarg.h>
#include <stdint.h>
#include <stdio.h>

#include "../../include/pulse.h"

namespace pulse {

inline thread_local char g_last_error[512];

inline int fail(int status, const char* fmt, ...) {
  va_list ap;
  va_start(ap, fmt);
  vsnprintf(g_last_error, sizeof g_last_error, fmt, ap);
  va_end(ap);
  return status;
}

inline int ok() {
  g_last_error[0] = '\0';
  return PULSE_OK;
}

inline bool aligned(const void* p, uintptr_t a) { return ((uintptr_t)p & (a - 1)) == 0; }
inline bool aligned16(const void* p) { return aligned(p, 16); }

inline int hip_status(hipError_t e, const char* what) {
  if (e != hipSuccess) return fail(PULSE_EHIP, "%s: %s", what, hipGetErrorString(e));
  return ok();
}

}  // namespace pulse
