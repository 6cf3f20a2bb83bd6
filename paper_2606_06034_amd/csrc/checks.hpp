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

// a device array of the call: its address and bytes
struct Span {
  const void* p;
  int64_t bytes;
};

// every array aligned; no output overlaps an input or another output, but for
// output same_out and input same_in where these are one array
inline int check_spans(const Span* in, int ni, const Span* out, int no, int same_out = -1,
                int same_in = -1) {
  for (int i = 0; i < ni; ++i)
    if (in[i].p && !aligned(in[i].p)) return GDN_ERR_ALIGN;
  for (int o = 0; o < no; ++o)
    if (out[o].p && !aligned(out[o].p)) return GDN_ERR_ALIGN;
  for (int o = 0; o < no; ++o) {
    for (int i = 0; i < ni; ++i) {
      if (o == same_out && i == same_in && out[o].p == in[i].p) continue;
      if (overlap(out[o].p, out[o].bytes, in[i].p, in[i].bytes)) return GDN_ERR_ALIAS;
    }
    for (int q = o + 1; q < no; ++q)
      if (overlap(out[o].p, out[o].bytes, out[q].p, out[q].bytes)) return GDN_ERR_ALIAS;
  }
  return GDN_OK;
}

inline bool valid_heads(int Hk, int Hv) { return Hk >= 0 && Hv >= 0 && (Hk ? Hv % Hk == 0 : Hv == 0); }

inline int hip_status(hipError_t e) {
  if (e == hipSuccess) return GDN_OK;
  if (e == hipErrorNotSupported) return GDN_ERR_UNSUPPORTED;
  return GDN_ERR_HIP;
}

}  // namespace checks
}  // namespace gdn
