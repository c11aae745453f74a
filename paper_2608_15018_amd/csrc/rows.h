// Checks of row strides and overlaps shared by the C-ABI sources (host only).
#pragma once

#include <cstdint>

#include "status.h"

namespace s2moe {

// Rows of `heads` heads, `ld` elements apart.
inline s2moe_status check_rows(const char* fn, const char* name, int64_t ld, int heads, int D,
                               int elt) {
  if (ld < (int64_t)heads * D)
    return fail(S2MOE_EINVAL, "%s: %s = %lld must be at least %d heads of %d", fn, name,
                (long long)ld, heads, D);
  if (ld > (int64_t)1 << 22)
    return fail(S2MOE_EUNSUPPORTED, "%s: %s = %lld exceeds 2^22 elements", fn, name, (long long)ld);
  if (ld * elt % 16 != 0)
    return fail(S2MOE_EINVAL, "%s: %s = %lld elements is not a multiple of 16 bytes", fn, name,
                (long long)ld);
  return S2MOE_OK;
}

// Whether rows of wa bytes every lda meet rows of wb bytes every ldb (n rows
// each): rows of one wider array may lie side by side.
inline bool rows_meet(const void* a, int64_t lda, int64_t wa, const void* b, int64_t ldb,
                      int64_t wb, int64_t n) {
  const int64_t x = (int64_t)reinterpret_cast<uintptr_t>(a);
  const int64_t y = (int64_t)reinterpret_cast<uintptr_t>(b);
  if (y >= x + (n - 1) * lda + wa || x >= y + (n - 1) * ldb + wb) return false;
  if (lda != ldb) return true;
  const int64_t at = ((y - x) % lda + lda) % lda;  // where b's rows start within a's period
  return at < wa || at + wb > lda;
}

// Whether two stretches of memory meet.
inline bool bytes_meet(const void* a, int64_t na, const void* b, int64_t nb) {
  const int64_t x = (int64_t)reinterpret_cast<uintptr_t>(a);
  const int64_t y = (int64_t)reinterpret_cast<uintptr_t>(b);
  return x < y + nb && y < x + na;
}

}  // namespace s2moe

// Arrays of 32-bit elements may start anywhere such an element may.
#define S2MOE_REQUIRE_INTS(p)                                                              \
  do {                                                                                     \
    if ((p) == nullptr) return fail(S2MOE_EINVAL, "%s: %s is NULL", fn, #p);               \
    if (!aligned(p, 4)) return fail(S2MOE_EINVAL, "%s: %s is not 4-byte aligned", fn, #p); \
  } while (0)
