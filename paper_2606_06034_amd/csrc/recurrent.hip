// recurrent.hip -- the gated delta rule token by token (decoding).
//
// Per sequence and value head, with the [dk, dv] state S in fp32,
//   S <- a S (a = e^g), u = beta (v - S^T k), S <- S + k u^T, o = scale S^T q.
// Both products with the state are taken from the state as it enters the
// token, S^T k and S^T q side by side, so that a token is one pass over S and
// one reduction over its rows:
//   u = beta (v - a S^T k),  o = scale (a S^T q + (k . q) u),
//   S <- a S + k u^T.
// Value columns are independent of each other, so a wave carries 32 of them
// for all dk rows with no exchange between waves.  Lane (r, c), r = lane / 8,
// c = lane % 8, holds rows r dk/8 .. and the 4 columns 4c .. in registers: a
// load of the wave covers whole 128-byte lines of 8 rows, and the sums over
// the rows end in three exchanges between lanes.
//
// Bound: the state is read and written once a call, 8 bytes for 7 flops a token.
// One token is HBM traffic: 256 sequences of 32 heads of 128 by 128, 1.08 GB, take
// 199 us, 5.4 TB/s.  A further token is 413 vector instructions of a wave, which
// take 432 slots of 4 cycles: 48 sequences of 21 heads of 128 by 64 (two waves a
// SIMD) take 10 us for a token each, 21 for 8 and 191 for 128, where the vector
// units are busy all the time and a token is 1.4 us.  1 to 8 tokens of them, 68 MB,
// take 19 us.
#include "lanes.hpp"
#include "launch.hpp"
#include "layer.hpp"
#include "tile16.hpp"

namespace gdn {

namespace {

template <int N>
__device__ __forceinline__ void load_n(float (&x)[N], const float* __restrict__ p) {
#pragma unroll
  for (int i = 0; i < N; i += 4) {
    const f32x4 t = *(const f32x4*)(p + i);
#pragma unroll
    for (int v = 0; v < 4; ++v) x[i + v] = t[v];
  }
}
template <int N>
__device__ __forceinline__ void load_n(float (&x)[N], const __bf16* __restrict__ p) {
#pragma unroll
  for (int i = 0; i < N; i += 8) {
    const bf16x8 t = *(const bf16x8*)(p + i);
#pragma unroll
    for (int v = 0; v < 8; ++v) x[i + v] = (float)t[v];
  }
}
__device__ __forceinline__ f32x4 load_4(const float* __restrict__ p) { return *(const f32x4*)p; }
__device__ __forceinline__ f32x4 load_4(const __bf16* __restrict__ p) {
  return __builtin_convertvector(*(const bf16x4*)p, f32x4);
}
__device__ __forceinline__ void store_4(float* p, f32x4 x) { *(f32x4*)p = x; }
__device__ __forceinline__ void store_4(__bf16* p, f32x4 x) {
  *(bf16x4*)p = __builtin_convertvector(x, bf16x4);
}

// sum over the 8 row groups (lanes 8, 16, 32 apart); every lane gets it
__device__ __forceinline__ float sum_groups(float x) {
  return sum_apart32(sum_apart16(sum_apart8(x)));
}

}  // namespace

// one wave a slice of 32 value columns
template <int DK, int DV, typename TIO>
__global__ __launch_bounds__(256) void k_recurrent(
    const TIO* __restrict__ Q, const TIO* __restrict__ K, const TIO* __restrict__ V,
    const float* __restrict__ beta, const float* __restrict__ g, const float* S0, TIO* __restrict__ O,
    float* Sfin, const int* __restrict__ slots, int n_states, const int* __restrict__ cu,
    uint32_t waves, int T, int Hk, int Hv, float scale) {
  constexpr int NR = DK / 8, NC = DV / 32;
  const uint32_t w = blockIdx.x * 4 + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  if (w >= waves) return;
  const int l = lane_id(), r0 = (l >> 3) * NR;
  const uint32_t sh = w / NC;
  const int s = (int)(sh / (uint32_t)Hv), h = (int)(sh - (uint32_t)s * (uint32_t)Hv);
  const int hk = h / (Hv / Hk);
  const int col = (int)(w - sh * NC) * 32 + 4 * (l & 7);
  int64_t t0 = (int64_t)s * T, n = T;
  if (cu) {
    const int a = cu[s], b = cu[s + 1];
    t0 = a;
    n = (a >= 0 && b <= T && b > a) ? b - a : 0;
  }
  const int slot = slots ? slots[s] : s;
  if (slot < 0 || slot >= n_states) {  // a padded sequence
    if (l < 8)
      for (int64_t t = t0; t < t0 + n; ++t) store_4(O + (t * Hv + h) * DV + col, zero4());
    return;
  }
  const int64_t sbase = ((int64_t)slot * Hv + h) * DK * DV + (int64_t)r0 * DV + col;
  if (n == 0 && (!Sfin || Sfin == S0)) return;
  f32x4 st[NR];
#pragma unroll
  for (int i = 0; i < NR; ++i) st[i] = S0 ? *(const f32x4*)(S0 + sbase + i * DV) : zero4();

  struct Tok {
    float k[NR], q[NR];
    f32x4 v;
    float b, g;
  };
  auto fetch = [&](Tok& x, int64_t t) __attribute__((always_inline)) {
    load_n(x.k, K + (t * Hk + hk) * DK + r0);
    load_n(x.q, Q + (t * Hk + hk) * DK + r0);
    x.v = load_4(V + (t * Hv + h) * DV + col);
    x.b = beta[t * Hv + h];
    x.g = g[t * Hv + h];
  };
  Tok x;
  if (n > 0) fetch(x, t0);
  for (int64_t t = t0; t < t0 + n; ++t) {
    Tok nx;
    fetch(nx, t + 1 < t0 + n ? t + 1 : t);
    f32x4 sk = zero4(), sq = zero4();
    float kq = 0.f;
#pragma unroll
    for (int i = 0; i < NR; ++i) {
      kq = __builtin_fmaf(x.k[i], x.q[i], kq);
#pragma unroll
      for (int v = 0; v < 4; ++v) {
        sk[v] = __builtin_fmaf(x.k[i], st[i][v], sk[v]);
        sq[v] = __builtin_fmaf(x.q[i], st[i][v], sq[v]);
      }
    }
    kq = sum_groups(kq);
#pragma unroll
    for (int v = 0; v < 4; ++v) {
      sk[v] = sum_groups(sk[v]);
      sq[v] = sum_groups(sq[v]);
    }
    const float a = expf(x.g);
    f32x4 u, o;
#pragma unroll
    for (int v = 0; v < 4; ++v) {
      u[v] = x.b * (x.v[v] - a * sk[v]);
      o[v] = scale * __builtin_fmaf(kq, u[v], a * sq[v]);
    }
#pragma unroll
    for (int i = 0; i < NR; ++i)
#pragma unroll
      for (int v = 0; v < 4; ++v) st[i][v] = __builtin_fmaf(x.k[i], u[v], a * st[i][v]);
    if (l < 8) store_4(O + (t * Hv + h) * DV + col, o);
    x = nx;
  }
  if (Sfin)
#pragma unroll
    for (int i = 0; i < NR; ++i) *(f32x4*)(Sfin + sbase + i * DV) = st[i];
}

hipError_t launch_recurrent(const void* Q, const void* K, const void* V, const float* beta,
                            const float* g, const float* S0, void* O, float* Sfin,
                            const int* slots, int n_states, const int* cu, int nseq, int T, int Hk,
                            int Hv, int dk, int dv, float scale, int dtype, hipStream_t st) {
  const int64_t waves = (int64_t)nseq * Hv * (dv / 32);
  const dim3 grid((unsigned)((waves + 3) / 4)), block(256);  // (checked to fit the grid)
  GDN_DK_SWITCH(dk, GDN_DV_SWITCH(dv, {
    if (dtype == 0)
      hipLaunchKernelGGL((k_recurrent<DK, DV, float>), grid, block, 0, st, (const float*)Q,
                         (const float*)K, (const float*)V, beta, g, S0, (float*)O, Sfin, slots,
                         n_states, cu, (uint32_t)waves, T, Hk, Hv, scale);
    else
      hipLaunchKernelGGL((k_recurrent<DK, DV, __bf16>), grid, block, 0, st, (const __bf16*)Q,
                         (const __bf16*)K, (const __bf16*)V, beta, g, S0, (__bf16*)O, Sfin, slots,
                         n_states, cu, (uint32_t)waves, T, Hk, Hv, scale);
    return hipGetLastError();
  }))
  return hipErrorNotSupported;
}

}  // namespace gdn
