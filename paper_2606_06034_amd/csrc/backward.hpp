// backward.hpp -- what the launches of the backward pass share (backward.hip,
// the per-chunk ones and the mathematics; walk.hip, the walks along the chunks).
#pragma once

#include "chunk.hpp"
#include "engine.hpp"
#include "forward.hpp"
#include "lanes.hpp"
#include "launch.hpp"
#include "layer.hpp"
#include "split.hpp"

namespace gdn {

constexpr int BC = 64;  // tokens a chunk

// Workspace of one (chunk, value head), in floats.  T lies as the terms (split.hpp)
// of the pair fragments of its row blocks, 3 KB a fragment (2 KB with fp32 inputs):
// (I, p) with 2p <= I; T^T is read from the same fragments, its pairs (I, p) have
// 2p + 1 >= I.
// X, R and dZ lie as column-form blocks, S and dS as row-form blocks (tile16.hpp),
// the 4 values of a lane side by side: 1 KB a block, read and written whole.
constexpr int TS = 768;
__host__ __device__ constexpr int blk_at(int I, int J, int NJ) { return (I * NJ + J) * 256; }
__host__ __device__ constexpr int t_slot(int I, int p) { return (I == 3 ? 4 : I) + p; }
__host__ __device__ constexpr int tt_slot(int I, int p) { return (I < 2 ? 2 * I : 2 + I) + p - I / 2; }
__host__ __device__ constexpr int64_t ws_T() { return 0; }
__host__ __device__ constexpr int64_t ws_rows() { return 6 * TS; }  // beta e^g e^{gl-g} g off
__host__ __device__ constexpr int64_t ws_R() { return ws_rows() + 5 * BC; }  // P^T dO, then dZ
__host__ __device__ constexpr int64_t ws_X(int dv) { return ws_R() + BC * dv; }
__host__ __device__ constexpr int64_t ws_S(int dv) { return ws_X(dv) + BC * dv; }
__host__ __device__ constexpr int64_t ws_dS(int dk, int dv) { return ws_S(dv) + dk * dv; }
__host__ __device__ constexpr int64_t ws_tile(int dk, int dv) { return ws_dS(dk, dv) + dk * dv; }

struct BwdArgs {
  const void *Q, *K, *V, *dO;
  const float *beta, *g, *S0, *dSf;
  void *dQ, *dK, *dV;
  float *dbeta, *dg, *dS0, *ws;
  const int* cu;
  int nseq, L;  // L: tokens a sequence, or all tokens where cu is given
  int nc;       // chunks a sequence (cu not given)
  int Hk, Hv, C;
  float scale;
  int gr;  // value heads a key head
};

// The chunks of sequence s lie at slots base(s), base(s) + 1, ...  Packed
// sequences: base(s) = cu[s] / 64 + s needs no table of its own, and
// base(s + 1) - base(s) is at least the sequence's chunks.  A sequence with
// offsets out of range is empty.
struct Seq {
  int64_t t0, base;
  int len;
  __device__ Seq(const BwdArgs& a, int s) {
    if (a.cu) {
      const int b = a.cu[s], e = a.cu[s + 1];
      const bool ok = b >= 0 && e >= b && e <= a.L;
      t0 = ok ? b : 0;
      len = ok ? e - b : 0;
      base = t0 / BC + s;
    } else {
      t0 = (int64_t)s * a.L;
      len = a.L;
      base = (int64_t)s * a.nc;
    }
  }
  __device__ int chunks() const { return (len + BC - 1) / BC; }
};

// first token and tokens (0: nothing to do) of the chunk at a slot
// (slots and heads of a launch fit 32 bits; a 64-bit division takes a thousand cycles)
__device__ __forceinline__ int chunk_at(const BwdArgs& a, uint32_t slot, int64_t& t0) {
  int s;
  if (a.cu) {
    // the last s with base(s) <= slot; a sequence that begins out of range has no chunks,
    // and its offset says nothing of the others': the next one in range is looked at
    int lo = 0, hi = a.nseq;
    while (hi - lo > 1) {
      const int mid = (lo + hi) >> 1;
      int at = mid, b = a.cu[at];
      while ((b < 0 || b > a.L) && ++at < hi) b = a.cu[at];
      if (at < hi && b / BC + at <= (int)slot) lo = at; else hi = mid;
    }
    s = lo;
  } else {
    s = (int)(slot / (uint32_t)a.nc);
  }
  const Seq q(a, s);
  const int64_t j = slot - q.base;
  if (j < 0 || j * BC >= q.len) return 0;
  t0 = q.t0 + j * BC;
  return min(BC, q.len - (int)j * BC);
}

__device__ __forceinline__ f32x4 mma16(f32x4 a, f32x4 b, f32x4 acc) {
#pragma unroll
  for (int v = 0; v < 4; ++v)
    acc = __builtin_amdgcn_mfma_f32_16x16x4f32(a[v], b[v], acc, 0, 0, 0);
  return acc;
}

// 4 values down a column (row stride ld), and 4 along a row
__device__ __forceinline__ f32x4 down4(const float* p, int ld) {
  return f32x4{p[0], p[ld], p[2 * ld], p[3 * ld]};
}
__device__ __forceinline__ f32x4 at4(const float* p) { return *(const f32x4*)p; }

// column-form block of rows r0 .. r0 + 15, columns from p's: as loaded (rows
// past m repeat the last one, so that no load is behind a branch), and its
// values (0 past m)
template <typename T> struct RawBlock { T v[4]; };
template <typename T>
__device__ __forceinline__ RawBlock<T> raw_block(const T* __restrict__ p, int64_t ld, int r0, int m) {
  RawBlock<T> x;
#pragma unroll
  for (int v = 0; v < 4; ++v) x.v[v] = p[min(r0 + 4 * lane_g() + v, m - 1) * ld + lane_c()];
  return x;
}
template <typename T>
__device__ __forceinline__ f32x4 block_of(const RawBlock<T>& x, int r0, int m) {
  f32x4 r;
#pragma unroll
  for (int v = 0; v < 4; ++v) r[v] = (float)x.v[v];
  if (m < r0 + 16)
#pragma unroll
    for (int v = 0; v < 4; ++v) r[v] = r0 + 4 * lane_g() + v < m ? r[v] : 0.f;
  return r;
}
template <typename T>
__device__ __forceinline__ f32x4 col_block(const T* __restrict__ p, int64_t ld, int r0, int m) {
  return block_of(raw_block(p, ld, r0, m), r0, m);
}

template <typename T> struct FragOf { typedef f32x4 type; };
template <> struct FragOf<__bf16> { typedef bf16x4 type; };

// the two walks of walk.hip: states first to last, their gradients last to first
hipError_t launch_walks(const BwdArgs& a, int dk, int dv, int dtype, hipStream_t st);

}  // namespace gdn
