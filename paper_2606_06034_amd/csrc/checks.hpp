// checks.hpp -- argument checks shared by the C entry points (internal).
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

#include "gdninv.h"

namespace gdn {
namespace checks {

// HIP's bounds of a 1-D launch of n workgroups of `block` work items
inline bool grid_ok(int64_t n, int block) {
  return n >= 0 && n <= 0x7fffffffLL && n * block <= 0xffffffffLL;
}

inline bool valid_C(int C) { return C == 16 || C == 32 || C == 64 || C == 128; }
inline bool valid_d(int d) { return d == 64 || d == 128; }
inline bool fdtype(int t) { return t == GDN_F32 || t == GDN_BF16; }
inline int64_t esize(int t) { return t == GDN_F32 ? 4 : (t == GDN_BF16 ? 2 : 1); }
inline bool aligned(const void* p) { return (reinterpret_cast<uintptr_t>(p) & 15u) == 0; }

// [p, p + bytes) and [q, q + qbytes) intersect
inline bool overlap(const void* p, int64_t bytes, const void* q, int64_t qbytes) {
  if (!p || !q || bytes <= 0 || qbytes <= 0) return false;
  const uintptr_t a = reinterpret_cast<uintptr_t>(p), b = reinterpret_cast<uintptr_t>(q);
  return a < b + (uintptr_t)qbytes && b < a + (uintptr_t)bytes;
}

inline int hip_status(hipError_t e) {
  if (e == hipSuccess) return GDN_OK;
  if (e == hipErrorNotSupported) return GDN_ERR_UNSUPPORTED;
  return GDN_ERR_HIP;
}

}  // namespace checks
}  // namespace gdn
