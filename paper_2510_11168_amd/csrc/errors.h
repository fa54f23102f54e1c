// Error texts of the C ABI, one per host thread, shared by the library's translation units.
#pragma once
#include <hip/hip_runtime.h>

#include <cstdarg>
#include <cstdio>

namespace elmo {

inline thread_local char g_err[512] = "";

inline int fail(int code, const char* fmt, ...) {
  va_list ap;
  va_start(ap, fmt);
  vsnprintf(g_err, sizeof g_err, fmt, ap);
  va_end(ap);
  return code;
}

inline int check_launch(const char* what) {
  hipError_t e = hipGetLastError();
  if (e != hipSuccess) return fail(-3, "launch of %s failed: %s", what, hipGetErrorString(e));
  return 0;
}

}  // namespace elmo

#define ELMO_HIP(call)                                                                             \
  do {                                                                                             \
    hipError_t e_ = (call);                                                                        \
    if (e_ != hipSuccess) return elmo::fail(-3, "%s failed: %s", #call, hipGetErrorString(e_));    \
  } while (0)
