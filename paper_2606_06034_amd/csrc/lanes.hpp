// lanes.hpp -- sums over the lanes of a wave on the cross-lane data paths of the
// vector unit (an exchange through LDS takes ten times as long).
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

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

// a lane and the one 16 (32) lanes away: x with the odd and the even rows of 16 (the
// halves of 32) exchanged between two copies, which then hold the one and the other.
// (Two copies for the compiler as well: of one value it takes the two results for one.)
__device__ __forceinline__ float sum_apart16(float x) {
  uint32_t a = __builtin_bit_cast(uint32_t, x), b = a;
  asm volatile("" : "+v"(b));
  const auto r = __builtin_amdgcn_permlane16_swap(a, b, false, false);
  return __builtin_bit_cast(float, (uint32_t)r[0]) + __builtin_bit_cast(float, (uint32_t)r[1]);
}
__device__ __forceinline__ float sum_apart32(float x) {
  uint32_t a = __builtin_bit_cast(uint32_t, x), b = a;
  asm volatile("" : "+v"(b));
  const auto r = __builtin_amdgcn_permlane32_swap(a, b, false, false);
  return __builtin_bit_cast(float, (uint32_t)r[0]) + __builtin_bit_cast(float, (uint32_t)r[1]);
}
__device__ __forceinline__ float sum_apart8(float x) { return x + lane_moved<0x128>(x); }

// over N = 32 or 64 neighbouring lanes
template <>
__device__ __forceinline__ float sum_lanes<32>(float x) {
  return sum_apart16(sum_lanes<16>(x));
}
template <>
__device__ __forceinline__ float sum_lanes<64>(float x) {
  return sum_apart32(sum_lanes<32>(x));
}

}  // namespace gdn
