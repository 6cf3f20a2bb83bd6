// norm.hpp -- what the norms' kernels share.
#pragma once

#include <hip/hip_runtime.h>

namespace gdn {

// 1 / (1 + e^-z).  The exponential and the reciprocal are the hardware's (1
// ulp, and |z| 6e-8 from the scaled argument): the exact ones made the
// vector operations as long as the memory traffic.
__device__ __forceinline__ float sigmoid(float z) {
  return __builtin_amdgcn_rcpf(1.f + __expf(-z));
}

}  // namespace gdn
