// split.hpp -- fp32 products on the bf16 matrix instructions.
//
// An fp32 value is the sum of three bf16 values to 2^-25 of itself (each takes
// 8 of the 24 bits of what the ones before left), and a product of bf16 values
// accumulated in fp32 is exact.  A product of a bf16 input with an fp32 value
// is then three matrix instructions, one of two fp32 values six (the terms
// below 2^-24 of the largest are left out), at 16 times the rate of the fp32
// instruction: 5.3 and 2.7 times its speed at its accuracy.  With fp32 inputs
// (F = f32x4) the same code runs on the fp32 instructions, one term each.
// An infinity, or a value that rounds to one in bf16, leaves a second term of inf -
// inf: products with it are NaN.
#pragma once

#include "tile16.hpp"

namespace gdn {

template <typename F> struct TermsOf { static constexpr int N = 3; };
template <> struct TermsOf<f32x4> { static constexpr int N = 1; };

// two values rounded to bf16 in one register (the low half a), and what is left
// of them.  (Taken apart by bits: from the converted values as such the compiler
// rounds the two apart and packs them afterwards, at twice the instructions.  Not
// by an instruction in assembly either: the wait states that a vector instruction
// needs after a matrix instruction on its registers are not kept for it.)
__device__ __forceinline__ uint32_t take2(float& a, float& b) {
  typedef float f32x2 __attribute__((ext_vector_type(2)));
  typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
  const uint32_t r = __builtin_bit_cast(uint32_t, __builtin_convertvector(f32x2{a, b}, bf16x2));
  a -= __builtin_bit_cast(float, r << 16);
  b -= __builtin_bit_cast(float, r & 0xffff0000u);
  return r;
}

// four values as terms
template <typename F> struct Half { F t[TermsOf<F>::N]; };
template <typename F>
__device__ __forceinline__ Half<F> split_half(f32x4 x) {
  Half<F> r;
  if constexpr (TermsOf<F>::N == 1) {
    r.t[0] = x;
  } else {
    typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));
    float a = x[0], b = x[1], c = x[2], d = x[3];
#pragma unroll
    for (int i = 0; i < 3; ++i) {
      const uint32_t lo = take2(a, b), hi = take2(c, d);
      r.t[i] = __builtin_bit_cast(bf16x4, u32x2{lo, hi});
    }
  }
  return r;
}

__device__ __forceinline__ Pair<bf16x4> join(bf16x4 a, bf16x4 b) {
  return Pair<bf16x4>{__builtin_shufflevector(a, b, 0, 1, 2, 3, 4, 5, 6, 7)};
}
__device__ __forceinline__ Pair<f32x4> join(f32x4 a, f32x4 b) { return Pair<f32x4>{a, b}; }

// a pair fragment as terms
template <typename F> struct Terms {
  Pair<F> t[TermsOf<F>::N];
};
template <typename F>
__device__ __forceinline__ Terms<F> split(f32x4 lo, f32x4 hi) {
  const Half<F> a = split_half<F>(lo), b = split_half<F>(hi);
  Terms<F> r;
#pragma unroll
  for (int i = 0; i < TermsOf<F>::N; ++i) r.t[i] = join(a.t[i], b.t[i]);
  return r;
}

// acc += x y, the input x exact; the smallest terms first
template <bool OUTQ, typename F>
__device__ __forceinline__ f32x4 mma_in(const Pair<F>& x, const Terms<F>& y, f32x4 acc) {
#pragma unroll
  for (int i = TermsOf<F>::N - 1; i >= 0; --i)
    acc = Pair<F>::template mma<OUTQ>(x, y.t[i], acc);
  return acc;
}
// the same for N left operands and one right one, term after term, so that
// neighbouring instructions do not wait for each other
template <bool OUTQ, int N, typename F>
__device__ __forceinline__ void mma_in(const Pair<F> (&x)[N], const Terms<F>& y, f32x4 (&acc)[N]) {
#pragma unroll
  for (int i = TermsOf<F>::N - 1; i >= 0; --i)
#pragma unroll
    for (int n = 0; n < N; ++n) acc[n] = Pair<F>::template mma<OUTQ>(x[n], y.t[i], acc[n]);
}
// acc += x y of two fp32 values, in two sums, one of the terms below the largest, so
// that half as many instructions wait for each other
template <bool OUTQ, typename F>
__device__ __forceinline__ void mma_both(const Terms<F>& x, const Terms<F>& y, f32x4& acc,
                                         f32x4& low) {
  if constexpr (TermsOf<F>::N == 1) {
    acc = Pair<F>::template mma<OUTQ>(x.t[0], y.t[0], acc);
  } else {
    low = Pair<F>::template mma<OUTQ>(x.t[0], y.t[2], low);
    acc = Pair<F>::template mma<OUTQ>(x.t[1], y.t[1], acc);
    low = Pair<F>::template mma<OUTQ>(x.t[2], y.t[0], low);
    acc = Pair<F>::template mma<OUTQ>(x.t[1], y.t[0], acc);
    low = Pair<F>::template mma<OUTQ>(x.t[0], y.t[1], low);
    acc = Pair<F>::template mma<OUTQ>(x.t[0], y.t[0], acc);
  }
}

// Terms in LDS: a slot is 64 lanes of one pair and term
template <typename T>
__device__ __forceinline__ T* slot_at(T* s, int pair, int term, int terms) {
  return s + (pair * terms + term) * 512;
}
template <typename F, typename T>
__device__ __forceinline__ void store_half(T* s, int pair, int hf, const Half<F>& x, int l) {
#pragma unroll
  for (int i = 0; i < TermsOf<F>::N; ++i) {
    T* p = slot_at(s, pair, i, TermsOf<F>::N);
    if constexpr (TermsOf<F>::N == 1)
      *(f32x4*)(p + 256 * hf + 4 * l) = x.t[i];
    else
      *(bf16x4*)(p + 8 * l + 4 * hf) = x.t[i];
  }
}
template <typename F, typename T>
__device__ __forceinline__ Terms<F> load_terms(const T* s, int pair, int l) {
  Terms<F> r;
#pragma unroll
  for (int i = 0; i < TermsOf<F>::N; ++i) {
    const T* p = slot_at(s, pair, i, TermsOf<F>::N);
    if constexpr (TermsOf<F>::N == 1)
      r.t[i] = Pair<F>{*(const f32x4*)(p + 4 * l), *(const f32x4*)(p + 256 + 4 * l)};
    else
      r.t[i].v = *(const bf16x8*)(p + 8 * l);
  }
  return r;
}
// Rows of an input in LDS, LD values apart: a pair along a row (slot s of lane
// (g, c): column c0 + 16 (s / 4) + 4g + s % 4 of row r0 + c) and one down the
// rows (row r0 + 16 (s / 4) + 4g + s % 4 of column c0 + c).  In bf16 the second
// is two of the transposing LDS reads: 16 lanes read a 4 x 16 block, lane i the
// four values at row i / 4, columns 4 (i % 4), and lane c receives column c.
template <int LD>
__device__ __forceinline__ Pair<f32x4> row_pair(const float* s, int r0, int c0, Lane ln) {
  const float* p = s + (r0 + ln.c()) * LD + c0 + 4 * ln.g();
  return join(*(const f32x4*)p, *(const f32x4*)(p + 16));
}
__device__ __forceinline__ bf16x4 read_transposed(const __bf16* p) {
  typedef short s16x4 __attribute__((ext_vector_type(4)));
  typedef __attribute__((address_space(3))) s16x4 lds_s16x4;
  return __builtin_bit_cast(bf16x4, __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4*)p));
}
template <int LD>
__device__ __forceinline__ Pair<bf16x4> col_pair(const __bf16* s, int r0, int c0, Lane ln) {
  const __bf16* p = s + (r0 + 4 * ln.g() + (ln.c() >> 2)) * LD + c0 + 4 * (ln.c() & 3);
  return join(read_transposed(p), read_transposed(p + 16 * LD));
}
template <int LD>
__device__ __forceinline__ Pair<f32x4> col_pair(const float* s, int r0, int c0, Lane ln) {
  const float* p = s + (r0 + 4 * ln.g()) * LD + c0 + ln.c();
  f32x4 a, b;
#pragma unroll
  for (int v = 0; v < 4; ++v) a[v] = p[v * LD], b[v] = p[(16 + v) * LD];
  return join(a, b);
}

// LDS writes before the barrier are visible after it; global memory is not
// waited for
__device__ __forceinline__ void lds_only_barrier() {
  __builtin_amdgcn_fence(__ATOMIC_RELEASE, "workgroup");
  __builtin_amdgcn_s_barrier();
  __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "workgroup");
}

// The same for a wave that only copies to LDS by DMA and has waited for the copies
// that the barrier is to publish: a fence would wait for all of them.
__device__ __forceinline__ void copier_barrier() {
  __builtin_amdgcn_sched_barrier(0);
  __builtin_amdgcn_s_barrier();
  __builtin_amdgcn_sched_barrier(0);
}

}  // namespace gdn
