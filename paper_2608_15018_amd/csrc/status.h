// Status codes and messages shared by the C-ABI sources (host only).
#pragma once

#include <hip/hip_runtime.h>

#include <cstdarg>
#include <cstdint>
#include <cstdio>
#include <string>

#include "s2moe.h"

namespace s2moe {

// Message of the calling thread's last failed call.
inline thread_local std::string g_last_error;

inline s2moe_status fail(s2moe_status st, const char* fmt, ...) {
  char buf[512];
  va_list ap;
  va_start(ap, fmt);
  vsnprintf(buf, sizeof(buf), fmt, ap);
  va_end(ap);
  g_last_error = buf;
  return st;
}

inline s2moe_status ok() {
  g_last_error.clear();
  return S2MOE_OK;
}

inline s2moe_status hip_status(const char* fn, hipError_t err) {
  if (err != hipSuccess) return fail(S2MOE_EHIP, "%s: %s", fn, hipGetErrorString(err));
  return ok();
}

inline bool aligned(const void* p, size_t a) {
  return (reinterpret_cast<uintptr_t>(p) & (a - 1)) == 0;
}

inline bool aligned16(const void* p) { return aligned(p, 16); }

}  // namespace s2moe

#define S2MOE_REQUIRE_PTR(p)                                                     \
  do {                                                                           \
    if ((p) == nullptr) return fail(S2MOE_EINVAL, "%s: %s is NULL", fn, #p);     \
    if (!aligned16(p)) return fail(S2MOE_EINVAL, "%s: %s is not 16-byte aligned", fn, #p); \
  } while (0)
