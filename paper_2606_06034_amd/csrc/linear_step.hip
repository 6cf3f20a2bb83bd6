// linear_step.hip -- linear attention with a decay for each head, token by token (decoding).
//
// Per sequence and value head, with the [dk, dv] state S in fp32,
//   S <- e^{g_t} S + k v^T,  o = scale S^T q.
// Value columns are independent of each other, so a wave carries NCOL of them for all dk rows
// in registers, with no exchange between waves: lane l holds dk NCOL / 256 rows of 4 columns,
// and the sums over the rows end in exchanges between lanes.
//
// Bound: HBM, the state is read and written once a call, 8 bytes for 5 flops a token: 198 us
// for 256 sequences of 32 heads of 128 x 128, 5.4 TB/s; 4.5 us for one of 16.
#include "lanes.hpp"
#include "launch.hpp"
#include "linear.hpp"
#include "tile16.hpp"

namespace gdn {

namespace {

template <int N>
__device__ __forceinline__ void load_run(float (&x)[N], const float* __restrict__ p) {
#pragma unroll
  for (int i = 0; i < N; ++i) x[i] = p[i];
}
template <int N>
__device__ __forceinline__ void load_run(float (&x)[N], const __bf16* __restrict__ p) {
  typedef __bf16 Vec __attribute__((ext_vector_type(N)));
  const Vec t = *(const Vec*)p;
#pragma unroll
  for (int i = 0; i < N; ++i) x[i] = (float)t[i];
}
__device__ __forceinline__ void store_run(float* p, f32x4 x) { *(f32x4*)p = x; }
__device__ __forceinline__ void store_run(__bf16* p, f32x4 x) {
  *(bf16x4*)p = __builtin_convertvector(x, bf16x4);
}

// over the lanes that hold the same columns: FROM, 2 FROM ... 32 lanes apart
template <int FROM>
__device__ __forceinline__ float sum_rows(float x) {
  if (FROM <= 2) x += __shfl_xor(x, 2);
  if (FROM <= 4) x += __shfl_xor(x, 4);
  x = sum_apart8(x);
  return sum_apart32(sum_apart16(x));
}

}  // namespace

template <int DK, int DV, int NCOL, typename T>
__global__ __launch_bounds__(256) void k_lin_step(
    const T* __restrict__ Q, const T* __restrict__ K, const T* __restrict__ V,
    const float* __restrict__ g, bool per_token, const float* S0, T* __restrict__ O, float* Sfin,
    const int* __restrict__ slots, int n_states, const int* __restrict__ cu, uint32_t waves, int T_,
    int Hk, int Hv, float scale) {
  constexpr int LC4 = NCOL / 4, NR = DK * LC4 / 64, NC = DV / NCOL;
  const uint32_t w = blockIdx.x * 4 + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  if (w >= waves) return;
  const int l = lane_id(), r0 = l / LC4 * NR;
  const uint32_t sh = w / NC;
  const int s = (int)(sh / (uint32_t)Hv), h = (int)(sh - (uint32_t)s * (uint32_t)Hv);
  const int hk = h / (Hv / Hk), col = (int)(w - sh * NC) * NCOL + 4 * (l % LC4);
  int64_t t0 = (int64_t)s * T_;
  int n = T_;
  if (cu) {
    const int a = cu[s], b = cu[s + 1];
    t0 = a;
    n = a >= 0 && b <= T_ && b > a ? b - a : 0;
  }
  const int slot = slots ? slots[s] : s;
  if (slot < 0 || slot >= n_states) {  // a padded sequence
    if (l < LC4)
      for (int64_t t = t0; t < t0 + n; ++t) store_run(O + (t * Hv + h) * DV + col, zero4());
    return;
  }
  if (n == 0 && (!Sfin || Sfin == S0)) return;
  const int64_t at = (((int64_t)slot * Hv + h) * DK + r0) * DV + col;
  f32x4 st[NR];
#pragma unroll
  for (int i = 0; i < NR; ++i) st[i] = S0 ? *(const f32x4*)(S0 + at + i * DV) : zero4();
  struct Tok {
    float k[NR], q[NR], v[4], a;
  };
  auto fetch = [&](Tok& x, int64_t t) __attribute__((always_inline)) {
    load_run(x.k, K + (t * Hk + hk) * DK + r0);
    load_run(x.q, Q + (t * Hk + hk) * DK + r0);
    load_run(x.v, V + (t * Hv + h) * DV + col);
    x.a = per_token ? g[t * Hv + h] : g[h];
  };
  Tok x;
  if (n > 0) fetch(x, t0);
  for (int i = 0; i < n; ++i) {
    const int64_t t = t0 + i;
    Tok nx;
    fetch(nx, i + 1 < n ? t + 1 : t);
    const float a = expf(x.a);
    f32x4 o = zero4();
#pragma unroll
    for (int u = 0; u < NR; ++u)
#pragma unroll
      for (int v = 0; v < 4; ++v) {
        st[u][v] = __builtin_fmaf(x.k[u], x.v[v], a * st[u][v]);
        o[v] = __builtin_fmaf(x.q[u], st[u][v], o[v]);
      }
#pragma unroll
    for (int v = 0; v < 4; ++v) o[v] = scale * sum_rows<LC4>(o[v]);
    if (l < LC4) store_run(O + (t * Hv + h) * DV + col, o);
    x = nx;
  }
  if (Sfin)
#pragma unroll
    for (int i = 0; i < NR; ++i) *(f32x4*)(Sfin + at + i * DV) = st[i];
}

hipError_t launch_linear_step(const void* Q, const void* K, const void* V, const float* g,
                              bool per_token, const float* S0, void* O, float* Sfin,
                              const int* slots, int n_states, const int* cu, int nseq, int T,
                              int Hk, int Hv, int dk, int dv, float scale, int dtype,
                              hipStream_t st) {
  constexpr int NCOL = kStepColumns;
  const int64_t waves = (int64_t)nseq * Hv * (dv / NCOL);
  const dim3 grid((unsigned)((waves + 3) / 4)), block(256);  // (checked to fit the grid)
  GDN_DK_SWITCH(dk, GDN_DV_SWITCH(dv, {
    if (dtype == 0)
      hipLaunchKernelGGL((k_lin_step<DK, DV, NCOL, float>), grid, block, 0, st, (const float*)Q,
                         (const float*)K, (const float*)V, g, per_token, S0, (float*)O, Sfin,
                         slots, n_states, cu, (uint32_t)waves, T, Hk, Hv, scale);
    else
      hipLaunchKernelGGL((k_lin_step<DK, DV, NCOL, __bf16>), grid, block, 0, st, (const __bf16*)Q,
                         (const __bf16*)K, (const __bf16*)V, g, per_token, S0, (__bf16*)O, Sfin,
                         slots, n_states, cu, (uint32_t)waves, T, Hk, Hv, scale);
    return hipGetLastError();
  }))
  return hipErrorNotSupported;
}

}  // namespace gdn
