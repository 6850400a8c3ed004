// Error reporting and argument checks shared by the C entry points.  Every check
// runs on the host before any launch; the message of a failed call is kept per
// thread for sa_last_error.
#pragma once

#include <hip/hip_runtime.h>
#include <stdarg.h>
#include <stddef.h>
#include <stdint.h>
#include <stdio.h>

#include <string>

#include "../../include/sa.h"

namespace sa {
namespace host {

inline std::string& last_error() {
  thread_local std::string text;
  return text;
}

inline int fail(int code, const char* fmt, ...) {
  char buf[512];
  va_list ap;
  va_start(ap, fmt);
  vsnprintf(buf, sizeof(buf), fmt, ap);
  va_end(ap);
  last_error() = buf;
  return code;
}

inline int ok() {
  last_error().clear();
  return SA_OK;
}

inline int check_launch(const char* what) {
  const hipError_t e = hipGetLastError();
  if (e != hipSuccess)
    return fail(SA_ERR_HIP, "%s: kernel launch failed: %s", what, hipGetErrorString(e));
  return ok();
}

inline bool aligned(const void* p, size_t a) {
  return (reinterpret_cast<uintptr_t>(p) % a) == 0;
}

inline int check_tensor(const char* fn, const char* name, const void* p, bool required,
                        size_t align) {
  if (p == nullptr) {
    if (required) return fail(SA_ERR_INVALID_ARG, "%s: %s is NULL", fn, name);
    return SA_OK;
  }
  if (!aligned(p, align))
    return fail(SA_ERR_INVALID_ARG, "%s: %s is not %zu-byte aligned", fn, name, align);
  return SA_OK;
}

inline int check_ws(const char* fn, const void* ws, size_t ws_bytes, size_t need) {
  if (ws_bytes < need)
    return fail(SA_ERR_WORKSPACE, "%s: workspace of %zu bytes is below the %zu required",
                fn, ws_bytes, need);
  if (need > 0 && ws == nullptr) return fail(SA_ERR_INVALID_ARG, "%s: ws is NULL", fn);
  if (need > 0 && !aligned(ws, 16))
    return fail(SA_ERR_INVALID_ARG, "%s: ws is not 16-byte aligned", fn);
  return SA_OK;
}

}  // namespace host
}  // namespace sa

#define SA_TRY(expr)          \
  do {                        \
    const int rc_ = (expr);   \
    if (rc_ != SA_OK) return rc_; \
  } while (0)
