// lanes.hpp -- sums over the lanes of a wave on the cross-lane data paths of the
// vector unit (an exchange through LDS takes ten times as long).
#pragma once

#include <hip/hip_runtime.h>

namespace gdn {

template <int CTRL>
__device__ __forceinline__ float lane_moved(float x) {
  return __builtin_bit_cast(
      float, __builtin_amdgcn_mov_dpp(__builtin_bit_cast(int, x), CTRL, 0xf, 0xf, true));
}

// over groups of N neighbouring lanes (N = 2, 4, ... 16); every lane gets its group's
template <int N>
__device__ __forceinline__ float sum_lanes(float x) {
  if (N >= 2) x += lane_moved<0xB1>(x);    // lane ^ 1
  if (N >= 4) x += lane_moved<0x4E>(x);    // lane ^ 2
  if (N >= 8) x += lane_moved<0x141>(x);   // 7 - lane, of 8
  if (N >= 16) x += lane_moved<0x140>(x);  // 15 - lane, of 16
  return x;
}
__device__ __forceinline__ float sum16(float x) { return sum_lanes<16>(x); }

// over N = 32 or 64 neighbouring lanes
template <>
__device__ __forceinline__ float sum_lanes<32>(float x) {
  x = sum_lanes<16>(x);
  return x + __shfl_xor(x, 16);
}
template <>
__device__ __forceinline__ float sum_lanes<64>(float x) {
  x = sum_lanes<32>(x);
  return x + __shfl_xor(x, 32);
}

}  // namespace gdn
