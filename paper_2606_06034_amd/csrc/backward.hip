// backward.hip -- gradients of the chunk-wise layer forward.
//
// With gamma the cumulative log-decay inside a chunk of 64 tokens, D_ij =
// e^{gamma_i - gamma_j} (i >= j), S the state entering the chunk and dS the
// gradient of the state leaving it, the forward pass is
//   A = stril(diag(beta) K K^T (.) D), T = (I + A)^-1, P = scale (Q K^T) (.) D,
//   X = V - diag(e^gamma) K S, Z = diag(beta) X, Y = T Z,
//   O = scale diag(e^gamma) Q S + P Y,
//   S' = e^gl S + K^T diag(e^{gl - gamma}) Y                (gl: the last gamma)
// and its reverse
//   dY = P^T dO + diag(e^{gl - gamma}) K dS,  dZ = T^T dY,  dV = dX = diag(beta) dZ,
//   dS_in = e^gl dS + Q^T diag(scale e^gamma) dO - K^T diag(e^gamma) dX,
//   dP = scale (dO Y^T) (.) D,  E = -stril((dZ Y^T) (.) D),  F = E K,
//   dQ = scale diag(e^gamma) dO S^T + dP K,
//   dK+ = diag(beta) (F - diag(e^gamma) dZ S^T),  R = diag(e^{gl - gamma}) Y dS^T,
//   dK- = dP^T Q + E^T diag(beta) K + R,  dK = dK+ + dK-,
//   dbeta_i = dZ_i . X_i + k_i . F_i,
//   dgamma_i = q_i . dQ_i + k_i . (dK+ - dK-)_i,
//   dgamma_last += sum_i k_i . R_i + e^gl <S, dS>.
// (The sums over i and j of dP (.) P and dA (.) A that gamma's gradient is made
// of are these dot products, so K K^T and Q K^T are not formed again; F is
// divided by nothing, so beta = 0 is an ordinary value.)
//
// Three launches: k_bwd_prep (every chunk: T, P^T dO), the walks along the chunks of
// walk.hip (the states entering the chunks, first to last, and the gradients of the
// states leaving them, last to first, side by side), k_bwd_grads (every chunk: the
// gradients).  The chunks here are always of 64 tokens, whatever chunk size
// the caller's g restarts at (16, 32 or 64): the result of the exact layer
// does not depend on it, and gamma is g plus the last g of the 64-chunk's
// earlier parts.
//
// Everything is formed in fp32, bf16 inputs too: the gradients of beta and g
// are differences of large sums, and their outputs are fp32.
#include "backward.hpp"

namespace gdn {

// ---- every chunk: T and P^T dO
// Wave w forms row block w of A and P, each block of A in row form and of P in column
// form, which is the row form of P^T, and inverts its own diagonal block; then it has
// block column w of T, and its part of the columns of P^T dO, P as terms.  What a
// thread needs of K, Q and dO is asked for at the start.
// (With T left to wave 0 and P^T dO in fp32 instructions the others waited for it: 79 us
// for 8192 tokens of 16 heads, 128 by 128 in bf16; now 50.  At 4 x 8192 tokens of 32
// value heads 324 us for 1.76 GB, 5.4 TB/s: HBM bounds it.)

// X = (I - L)^-1 of a strictly lower 16 x 16 block, lr its row form, in both forms: with
// O_k the entries of L that join two blocks of size 2^k into one of size 2^(k+1),
// X_1 = I + O_0 and X_{k+1} = X_k + X_k O_k X_k, exact since O_k X_k O_k = 0.
__device__ __forceinline__ void inverse16(const f32x4& lr, f32x4& xr, f32x4& xc, Lane ln) {
  const int g = ln.g(), c = ln.c();
  const f32x4 lc = mma16(lr, eye4(ln), zero4());
  xr = xc = eye4(ln);
#pragma unroll
  for (int v = 0; v < 4; ++v) {
    if (in_level(c, 4 * g + v, 0)) xr[v] += lr[v];
    if (in_level(4 * g + v, c, 0)) xc[v] += lc[v];
  }
#pragma unroll
  for (int k = 1; k < 4; ++k) {
    f32x4 oc;
#pragma unroll
    for (int v = 0; v < 4; ++v) oc[v] = in_level(4 * g + v, c, k) ? lc[v] : 0.f;
    const f32x4 t = mma16(oc, xr, zero4());  // X_k O_k, row form
    const f32x4 n = mma16(t, xc, xc);
    xr = mma16(xc, t, xr);
    xc = n;
  }
}

template <int DK, int DV, typename T>
__global__ __launch_bounds__(256) void k_bwd_prep(const BwdArgs a) {
  typedef typename FragOf<T>::type F;
  constexpr int E = 16 / sizeof(T), LDV = DV + E, NQ = DK / 32, CPR = DV / E, ON = BC * CPR / 256;
  constexpr int NJ = DV / 16, TW = TS * 4 / sizeof(T);  // TW: values of T a slot of T
  typedef T Vec __attribute__((ext_vector_type(E)));
  __shared__ __attribute__((aligned(16))) float sA[10 * 256];
  __shared__ __attribute__((aligned(16))) T sP[6 * TermsOf<F>::N * 512], sO[BC * LDV];
  __shared__ __attribute__((aligned(16))) float sr[5][BC];
  const uint32_t slot = blockIdx.x / (uint32_t)a.Hv;
  const int h = (int)(blockIdx.x - slot * (uint32_t)a.Hv), hk = h / a.gr;
  int64_t t0 = 0;
  const int m = chunk_at(a, slot, t0);
  if (m == 0) return;
  float* ws = a.ws + (int64_t)blockIdx.x * ws_tile(DK, DV);
  const int wv = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const Lane ln = lane_here();
  const int l = ln.id, g = ln.g(), c = ln.c();
  Pair<F> q[NQ], k[NQ], kj[3][NQ];
  {
    const uint32_t ld = (uint32_t)a.Hk * DK;
    const T* Kp = (const T*)a.K + (t0 * a.Hk + hk) * DK;
    const T* Qp = (const T*)a.Q + (t0 * a.Hk + hk) * DK;
    auto rows = [&](Pair<F>(&x)[NQ], const T* p, int I) __attribute__((always_inline)) {
      const uint32_t at = min(16 * I + c, m - 1) * ld + 8 * g;
#pragma unroll
      for (int s = 0; s < NQ; ++s) x[s] = load_row8<F>(p + (at + 32 * s));
    };
    rows(k, Kp, wv);
    rows(q, Qp, wv);
#pragma unroll
    for (int J = 0; J < 3; ++J)
      if (J < wv) rows(kj[J], Kp, J);
  }
  Vec o[ON];
  {
    const T* dO = (const T*)a.dO + (t0 * a.Hv + h) * DV;
    const uint32_t ld = (uint32_t)a.Hv * DV;
#pragma unroll
    for (int i = 0; i < ON; ++i) {
      const int at = threadIdx.x + 256 * i;
      o[i] = *(const Vec*)(dO + (min(at / CPR, m - 1) * ld + at % CPR * E));
    }
  }
  if (threadIdx.x < BC) {
    const int r = threadIdx.x, rr = r < m ? r : m - 1;
    const float* gp = a.g + t0 * a.Hv + h;
    // the decay up to the parts (of C tokens) of row rr and of the last row
    float off = 0.f, offl = 0.f;
    for (int e = a.C; e < BC; e += a.C) {
      const float x = e < m ? gp[(int64_t)(e - 1) * a.Hv] : 0.f;
      if (rr >= e) off += x;
      offl += x;
    }
    const float gr = gp[(int64_t)rr * a.Hv], gl = gp[(int64_t)(m - 1) * a.Hv];
    sr[0][r] = r < m ? a.beta[(t0 + r) * a.Hv + h] : 0.f;
    sr[1][r] = expf(gr + off);
    sr[2][r] = expf((gl - gr) + (offl - off));
    sr[3][r] = gr;
    sr[4][r] = off;
#pragma unroll
    for (int k = 0; k < 5; ++k) ws[ws_rows() + k * BC + r] = sr[k][r];
  }
#pragma unroll
  for (int i = 0; i < ON; ++i) {
    const int at = threadIdx.x + 256 * i;
    *(Vec*)(sO + at / CPR * LDV + at % CPR * E) = at / CPR < m ? o[i] : Vec{};
  }
  __syncthreads();
  f32x4 xc;  // the inverse of this wave's diagonal block, column form
  {
    auto block = [&](const Pair<F>(&x)[NQ], int J) __attribute__((always_inline)) {
      f32x4 kk = zero4(), qk = zero4();
#pragma unroll
      for (int s = 0; s < NQ; ++s) {
        kk = Pair<F>::template mma<true>(k[s], x[s], kk);
        qk = Pair<F>::template mma<false>(q[s], x[s], qk);
      }
      // (rows past the chunk's last repeat it; beta is 0 there, P is masked)
#pragma unroll
      for (int v = 0; v < 4; ++v) {
        const int e = 4 * g + v;
        const int ia = 16 * wv + c, ja = 16 * J + e, ip = 16 * wv + e, jp = 16 * J + c;
        const float da = __expf((sr[3][ia] - sr[3][ja]) + (sr[4][ia] - sr[4][ja]));
        const float dp = __expf((sr[3][ip] - sr[3][jp]) + (sr[4][ip] - sr[4][jp]));
        kk[v] = ia > ja ? -sr[0][ia] * kk[v] * da : 0.f;
        qk[v] = ip >= jp && ip < m ? a.scale * qk[v] * dp : 0.f;
      }
      store_half<F>(sP, tt_slot(J, wv >> 1), wv & 1, split_half<F>(qk), l);
      return kk;
    };
#pragma unroll
    for (int J = 0; J < 3; ++J)
      if (J < wv) *(f32x4*)(sA + bidx(wv, J) * 256 + 4 * l) = block(kj[J], J);
    f32x4 xr;
    inverse16(block(k, wv), xr, xc, ln);
    *(f32x4*)(sA + bidx(wv, wv) * 256 + 4 * l) = xr;
    T* const Tw = (T*)(ws + ws_T());
    store_half<F>(Tw + TW * t_slot(wv, wv >> 1), 0, wv & 1, split_half<F>(xr), l);
    if (wv & 1) {  // the blocks beside the diagonal that their pairs take along: zeros
      store_half<F>(Tw + TW * t_slot(wv - 1, wv >> 1), 0, 1, split_half<F>(zero4()), l);
      store_half<F>(sP, tt_slot(wv, wv >> 1), 0, split_half<F>(zero4()), l);
    }
  }
  __syncthreads();
  {
    // X_IJ = X_II sum_{K = J}^{I - 1} L_IK X_KJ, J = w, rows in order
    f32x4 X[4] = {xc, zero4(), zero4(), zero4()};  // X_{w + d, w}, column form
#pragma unroll
    for (int d = 1; d < 4; ++d) {
      const int I = wv + d;
      if (I > 3) continue;
      f32x4 x = zero4();
#pragma unroll
      for (int e = 0; e < d; ++e) x = mma16(at4(sA + bidx(I, wv + e) * 256 + 4 * l), X[e], x);
      const f32x4 xi = at4(sA + bidx(I, I) * 256 + 4 * l);
      X[d] = mma16(xi, x, zero4());
      store_half<F>((T*)(ws + ws_T()) + TW * t_slot(I, wv >> 1), 0, wv & 1,
                    split_half<F>(mma16(x, xi, zero4())), l);
    }
  }
  {
    Terms<F> P[6];
#pragma unroll
    for (int i = 0; i < 6; ++i) P[i] = load_terms<F>(sP, i, l);
    // wave 3 has had no products of T, wave 0 the most
    const int J1 = (wv + 1) * (NJ / 4) - (wv < 3);
#pragma unroll 1
    for (int J = wv * (NJ / 4) - (wv > 0); J < J1; ++J) {
      f32x4 x[4];
#pragma unroll
      for (int I = 0; I < 4; ++I) x[I] = zero4();
#pragma unroll
      for (int p = 0; p < 2; ++p) {
        const Pair<F> y = col_pair<LDV>(sO, 32 * p, 16 * J, ln);
#pragma unroll
        for (int t = TermsOf<F>::N - 1; t >= 0; --t)
#pragma unroll
          for (int I = 0; I < 4; ++I)
            if (p >= I / 2) x[I] = Pair<F>::template mma<false>(P[tt_slot(I, p)].t[t], y, x[I]);
      }
#pragma unroll
      for (int I = 0; I < 4; ++I) *(f32x4*)(ws + ws_R() + blk_at(I, J, NJ) + 4 * l) = x[I];
    }
  }
}

// dg of row r from gamma's gradient: the last g of a part of C tokens is in the gamma of
// every later row
__device__ __forceinline__ float part_sum(const float* dgamma, int r, int m, int C) {
  float dg = dgamma[r];
  if (C < BC && r % C == C - 1)
    for (int i = r + 1; i < m; ++i) dg += dgamma[i];
  return dg;
}

// ---- every chunk: dQ, dK, dbeta, dg; the value heads of a key head in turn
// Eight waves.  Wave w has the 32 feature columns 32 (w % (DK / 32)) of dQ and dK
// for NR row blocks of the chunk.  dO, dZ and Y lie in LDS as pair fragments along
// the value columns (one form serves as left operand and, transposed, as right
// one); S and dS come from memory as right operands, each value split into
// terms by the waves that use it.  The blocks of dP and E wait in registers until the
// products with the states are done, and then take the place of dO and dZ.
// Bound: the instructions of two waves a SIMD (a workgroup fills a CU's LDS), which are in
// the same phase, so that one's vector work hides little of the other's matrix work:
// 20 us a chunk.  (Asking for the next chunk's operands a chunk ahead, and
// the two waves at different priorities, changed nothing.)
template <int DK, int DV, typename T>
struct Grads {
  typedef typename FragOf<T>::type F;
  static constexpr int NT = TermsOf<F>::N, NP = DV / 32;  // NP: pairs along the value columns
  static constexpr int NC = DK / 32, RG = 8 / NC, NR = 4 / RG;
  static constexpr int LDK = DK + 16 / sizeof(T);
  // LDS, in values of T: T, dO, dZ and Y; later dP and E along their rows and down
  // them, and the rows of K and Q
  static constexpr int oT = 0, oO = oT + 6 * NT * 512, oZ = oO + 4 * NP * 512;
  static constexpr int oY = oZ + 4 * NP * NT * 512, oEnd = oY + 4 * NP * NT * 512;
  static constexpr int oPr = 0, oPc = 6 * NT * 512, oEr = 2 * oPc, oEc = 3 * oPc, oK = 4 * oPc;
  static constexpr int oQ = oK + BC * LDK, oEnd2 = oQ + BC * LDK;
  static constexpr int SIZE = oEnd2 > oEnd ? oEnd2 : oEnd;
};

template <int DK, int DV, typename T>
__global__ __launch_bounds__(512) void k_bwd_grads(const BwdArgs a) {
  typedef Grads<DK, DV, T> G;
  typedef typename G::F F;
  constexpr int NT = G::NT, NP = G::NP, NR = G::NR, LDK = G::LDK;
  constexpr int E = 16 / sizeof(T), NJ = DV / 16, RY = 8 / NJ, TB = 16 * 20;
  typedef T Vec __attribute__((ext_vector_type(E)));
  __shared__ __attribute__((aligned(16))) T sm[G::SIZE];
  __shared__ __attribute__((aligned(16))) float sr[5][BC];
  __shared__ __attribute__((aligned(16))) float tr[8][2 * TB];
  __shared__ __attribute__((aligned(16))) float sdb[NJ][BC];
  __shared__ float red[2][G::NC][BC], sdg[BC], send[8];
  const uint32_t slot = blockIdx.x / (uint32_t)a.Hk;
  const int hk = (int)(blockIdx.x - slot * (uint32_t)a.Hk), gr = a.gr;
  int64_t t0 = 0;
  const int m = chunk_at(a, slot, t0);
  if (m == 0) return;
  const int wv = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int col = 32 * (wv % G::NC), I0 = wv / G::NC * NR;  // this wave's columns and row blocks
  const int64_t kld = (int64_t)a.Hk * DK, kat = (t0 * a.Hk + hk) * DK;
  const int64_t vld = (int64_t)a.Hv * DV;

  for (int h = hk * gr; h < (hk + 1) * gr; ++h) {
    // A value of its own in every turn: the LDS and memory offsets made from it
    // are formed where they are used.  Formed before the loop, some hundred of
    // them went to scratch, and their reloads were most of the kernel's time.
    int tid = threadIdx.x;
    asm volatile("" : "+v"(tid));
    const Lane ln{tid & 63};
    const int l = ln.id, g = ln.g(), c = ln.c();
    float* ws = a.ws + ((int64_t)slot * a.Hv + h) * ws_tile(DK, DV);
    const float* S = ws + ws_S(DV) + blk_at(col / 16, 0, NJ) + 4 * l;
    const float* dS = ws + ws_dS(DK, DV) + blk_at(col / 16, 0, NJ) + 4 * l;
    // S and dS of a pair of value column blocks
    struct States {
      f32x4 s[2][2], d[2][2];
    };
    auto states = [&](States& x, int p) __attribute__((always_inline)) {
#pragma unroll
      for (int b = 0; b < 2; ++b)
#pragma unroll
        for (int hf = 0; hf < 2; ++hf) {
          x.s[b][hf] = at4(S + blk_at(b, 2 * p + hf, NJ));
          x.d[b][hf] = at4(dS + blk_at(b, 2 * p + hf, NJ));
        }
    };
    // ---- T, dO and dZ into fragments, Z, and dZ . X
    const int J = wv % NJ;
    Terms<F> z[2];
    {
      f32x4 xb[4], zb[4];
#pragma unroll
      for (int I = 0; I < 4; ++I) {
        xb[I] = at4(ws + ws_X(DV) + blk_at(I, J, NJ) + 4 * l);
        zb[I] = at4(ws + ws_R() + blk_at(I, J, NJ) + 4 * l);
      }
      constexpr int PR = DV / 4;  // 4-value pieces a row, one of a fragment's lane each
      const T* dO = (const T*)a.dO + (t0 * a.Hv + h) * DV;
      F o[BC * PR / 512];
#pragma unroll
      for (int i = 0; i < BC * PR / 512; ++i) {
        const int at = tid + 512 * i, r = at / PR;
        o[i] = *(const F*)(dO + min(r, m - 1) * vld + at % PR * 4);
      }
      constexpr int TN = 6 * NT * 512 / E;  // 16-byte pieces of T
      Vec tv[(TN + 511) / 512];
#pragma unroll
      for (int i = 0; i < (TN + 511) / 512; ++i) {
        const int at = min(tid + 512 * i, TN - 1), sl = at / (NT * 512 / E);
        tv[i] = *(const Vec*)((const T*)(ws + ws_T() + TS * sl) + (at - sl * (NT * 512 / E)) * E);
      }
      if (tid < 5 * BC) (&sr[0][0])[tid] = ws[ws_rows() + tid];
      f32x4 bt[4];
#pragma unroll
      for (int I = 0; I < 4; ++I) bt[I] = at4(ws + ws_rows() + 16 * I + 4 * g);
      __builtin_amdgcn_sched_barrier(0);
#pragma unroll
      for (int p = 0; p < 2; ++p) z[p] = split<F>(bt[2 * p] * xb[2 * p], bt[2 * p + 1] * xb[2 * p + 1]);
      // dZ in row form by way of LDS, two blocks a turn
      float* t = tr[wv];
#pragma unroll
      for (int n = 0; n < 4 / RY; n += 2) {
#pragma unroll
        for (int k = 0; k < 2; ++k) {
          const int I = (n + k) * RY + wv / NJ;
          const f32x4 zv = wv / NJ ? zb[(n + k) * RY + RY - 1] : zb[(n + k) * RY];
          const f32x4 xv = wv / NJ ? xb[(n + k) * RY + RY - 1] : xb[(n + k) * RY];
          f32x4 dot;
#pragma unroll
          for (int v = 0; v < 4; ++v) {
            t[TB * k + (4 * g + v) * 20 + c] = zv[v];
            dot[v] = sum16(xv[v] * zv[v]);
          }
          if (c == 0) *(f32x4*)(sdb[J] + 16 * I + 4 * g) = dot;
        }
        lds_sync<true>();
#pragma unroll
        for (int k = 0; k < 2; ++k) {
          const int I = (n + k) * RY + wv / NJ;
          store_half<F>(sm + G::oZ, I * NP + (J >> 1), J & 1,
                        split_half<F>(at4(t + TB * k + c * 20 + 4 * g)), l);
        }
        lds_sync<true>();
      }
#pragma unroll
      for (int i = 0; i < BC * PR / 512; ++i) {
        const int at = tid + 512 * i, r = at / PR, e = at % PR;
        const int to = 16 * (e & 3) + (r & 15), hf = (e >> 2) & 1;
        T* po = sm + G::oO + ((r >> 4) * NP + (e >> 3)) * 512;
        *(F*)(sizeof(T) == 4 ? po + 256 * hf + 4 * to : po + 8 * to + 4 * hf) = r < m ? o[i] : F{};
      }
#pragma unroll
      for (int i = 0; i < (TN + 511) / 512; ++i)
        if (tid + 512 * i < TN) *(Vec*)(sm + G::oT + (tid + 512 * i) * E) = tv[i];
    }
    __syncthreads();
    // ---- Y = T Z: value column block J of the rows I % RY; the terms of each kind side
    // by side, so that neighbouring instructions do not wait for each other
    constexpr int tx[6] = {0, 1, 2, 1, 0, 0}, ty[6] = {2, 1, 0, 0, 1, 0};
    {
      constexpr int RN = 4 / RY;
      f32x4 y[RN], yl[RN];
#pragma unroll
      for (int n = 0; n < RN; ++n) y[n] = yl[n] = zero4();
#pragma unroll
      for (int p = 0; p < 2; ++p) {
        Terms<F> ts[RN];
#pragma unroll
        for (int n = 0; n < RN; ++n) {
          const int I = n * RY + wv / NJ;  // (2 p <= I where p <= n RY / 2)
          if (p <= n * RY / 2) ts[n] = load_terms<F>(sm + G::oT, t_slot(I, p), l);
        }
#pragma unroll
        for (int k = NT == 1 ? 5 : 0; k < 6; ++k)
#pragma unroll
          for (int n = 0; n < RN; ++n)
            if (p <= n * RY / 2) {
              f32x4& acc = k & 1 ? y[n] : yl[n];
              acc = Pair<F>::template mma<true>(ts[n].t[NT == 1 ? 0 : tx[k]], z[p].t[NT == 1 ? 0 : ty[k]],
                                                acc);
            }
      }
#pragma unroll
      for (int n = 0; n < RN; ++n)
        store_half<F>(sm + G::oY, (n * RY + wv / NJ) * NP + (J >> 1), J & 1,
                      split_half<F>(y[n] + yl[n]), l);
    }
    States st;
    states(st, 0);
    __syncthreads();
    // ---- dP and E, a lower block each; an E block costs as much as two of dP
    struct Blk {
      int kind, I, J;  // kind: 0 dP, 1 E, -1 none (then any block)
    };
    auto block = [&](int i) __attribute__((always_inline)) {
      // waves 0, 1: two of E; the others one of E and two (6, 7: one) of dP
      int kind, n;
      if (wv < 2) {
        kind = i < 2 ? 1 : -1;
        n = 2 * wv + i;
      } else if (i == 0) {
        kind = 1;
        n = wv + 2;
      } else {
        kind = wv < 6 || i == 1 ? 0 : -1;
        n = wv < 6 ? 2 * (wv - 2) + i - 1 : wv + 2;
      }
      n = min(n, 9);
      const int I = n < 1 ? 0 : n < 3 ? 1 : n < 6 ? 2 : 3;
      return Blk{kind, I, n - I * (I + 1) / 2};
    };
    f32x4 pe[3], pl[3];
    Blk bk[3];
#pragma unroll
    for (int i = 0; i < 3; ++i) {
      bk[i] = block(i);
      pe[i] = pl[i] = zero4();
    }
#pragma unroll 1
    for (int p = 0; p < NP; ++p) {
      // the first is an E; the second another (waves 0, 1) or a dP, the third a dP
      Terms<F> e0 = load_terms<F>(sm + G::oZ, bk[0].I * NP + p, l);
      Terms<F> y0 = load_terms<F>(sm + G::oY, bk[0].J * NP + p, l);
      if (wv < 2) {
        const Terms<F> e1 = load_terms<F>(sm + G::oZ, bk[1].I * NP + p, l);
        const Terms<F> y1 = load_terms<F>(sm + G::oY, bk[1].J * NP + p, l);
        mma_both<false>(e0, y0, pe[0], pl[0]);
        mma_both<false>(e1, y1, pe[1], pl[1]);
      } else {
        const Pair<F> o1 = slot_load<F>(sm + G::oO + (bk[1].I * NP + p) * 512, l);
        const Terms<F> y1 = load_terms<F>(sm + G::oY, bk[1].J * NP + p, l);
        mma_both<false>(e0, y0, pe[0], pl[0]);
        pe[1] = mma_in<false>(o1, y1, pe[1]);
        if (bk[2].kind == 0)
          pe[2] = mma_in<false>(slot_load<F>(sm + G::oO + (bk[2].I * NP + p) * 512, l),
                                load_terms<F>(sm + G::oY, bk[2].J * NP + p, l), pe[2]);
      }
    }
#pragma unroll
    for (int i = 0; i < 3; ++i)
#pragma unroll
      for (int v = 0; v < 4; ++v) {
        const int r = 16 * bk[i].I + 4 * g + v, j = 16 * bk[i].J + c;
        const float x = pe[i][v] + pl[i][v];
        const float d = r >= j ? __expf((sr[3][r] - sr[3][j]) + (sr[4][r] - sr[4][j])) : 0.f;
        pe[i][v] = bk[i].kind == 1 ? (r > j ? -x * d : 0.f) : a.scale * x * d;
      }
    // ---- dO S^T, dZ S^T, Y dS^T and <S, dS>
    constexpr int CPR = DK / E, KN = BC * CPR / 512;
    Vec kv[KN], qv[KN];
#pragma unroll
    for (int i = 0; i < KN; ++i) {
      const int at = tid + 512 * i, r = at / CPR;
      const int64_t from = kat + min(r, m - 1) * kld + at % CPR * E;
      kv[i] = *(const Vec*)((const T*)a.K + from);
      qv[i] = *(const Vec*)((const T*)a.Q + from);
    }
    f32x4 dq[2][NR], zs[2][NR], yd[2][NR];
    float ss = 0.f;
#pragma unroll
    for (int b = 0; b < 2; ++b)
#pragma unroll
      for (int i = 0; i < NR; ++i) dq[b][i] = zs[b][i] = yd[b][i] = zero4();
#pragma unroll 1
    for (int p = 0; p < NP; ++p) {
      Terms<F> sv[2], dv[2];
#pragma unroll
      for (int b = 0; b < 2; ++b) {
#pragma unroll
        for (int hf = 0; hf < 2; ++hf)
#pragma unroll
          for (int v = 0; v < 4; ++v) ss = __builtin_fmaf(st.s[b][hf][v], st.d[b][hf][v], ss);
        sv[b] = split<F>(st.s[b][0], st.s[b][1]);
        dv[b] = split<F>(st.d[b][0], st.d[b][1]);
      }
      states(st, p + 1 < NP ? p + 1 : p);
#pragma unroll
      for (int i = 0; i < NR; ++i) {
        const int at = (I0 + i) * NP + p;
        const Pair<F> o = slot_load<F>(sm + G::oO + at * 512, l);
        const Terms<F> z = load_terms<F>(sm + G::oZ, at, l), y = load_terms<F>(sm + G::oY, at, l);
#pragma unroll
        for (int k = NT == 1 ? 5 : 0; k < 6; ++k)
#pragma unroll
          for (int b = 0; b < 2; ++b) {
            const int kx = NT == 1 ? 0 : tx[k], ky = NT == 1 ? 0 : ty[k];
            zs[b][i] = Pair<F>::template mma<true>(z.t[kx], sv[b].t[ky], zs[b][i]);
            yd[b][i] = Pair<F>::template mma<true>(y.t[kx], dv[b].t[ky], yd[b][i]);
            if (k >= 6 - NT)
              dq[b][i] = Pair<F>::template mma<true>(o, sv[b].t[5 - k], dq[b][i]);
          }
      }
    }
    __syncthreads();
    // ---- K and Q, and dP and E as left operands: along their rows, and down them (E
    // with beta)
#pragma unroll
    for (int i = 0; i < KN; ++i) {
      const int at = tid + 512 * i, r = at / CPR, e = at % CPR * E;
      *(Vec*)(sm + G::oK + r * LDK + e) = r < m ? kv[i] : Vec{};
      *(Vec*)(sm + G::oQ + r * LDK + e) = r < m ? qv[i] : Vec{};
    }
#pragma unroll
    for (int i = 0; i < 3; ++i) {
      const Blk k = bk[i];
      if (k.kind < 0) continue;
      T* rows = sm + (k.kind ? G::oEr : G::oPr);
      T* cols = sm + (k.kind ? G::oEc : G::oPc);
      const f32x4 x = pe[i];
      float* t = tr[wv];
#pragma unroll
      for (int v = 0; v < 4; ++v) t[(4 * g + v) * 20 + c] = x[v];
      lds_sync<true>();
      store_half<F>(rows, t_slot(k.I, k.J >> 1), k.J & 1, split_half<F>(at4(t + c * 20 + 4 * g)), l);
      lds_sync<true>();
      store_half<F>(cols, tt_slot(k.J, k.I >> 1), k.I & 1,
                    split_half<F>(k.kind ? at4(&sr[0][16 * k.I + 4 * g]) * x : x), l);
      if (k.I == k.J) {  // the block beside the diagonal that its pair takes along: zeros
        if (k.I % 2 == 0)
          store_half<F>(rows, t_slot(k.I, k.I >> 1), 1, split_half<F>(zero4()), l);
        else
          store_half<F>(cols, tt_slot(k.I, k.I >> 1), 0, split_half<F>(zero4()), l);
      }
    }
    __syncthreads();
    // ---- the rest of dQ and dK, and the sums along their rows
    // right operands K and Q: pairs of token blocks, this wave's two column blocks
    Pair<F> kf[2][2], qf[2][2];
#pragma unroll
    for (int b = 0; b < 2; ++b)
#pragma unroll
      for (int p = 0; p < 2; ++p) {
        kf[b][p] = col_pair<LDK>(sm + G::oK, 32 * p, col + 16 * b, ln);
        qf[b][p] = col_pair<LDK>(sm + G::oQ, 32 * p, col + 16 * b, ln);
      }
    // The sums over the value heads of a key head, in the place of the first one's
    // states (which nothing reads any more); the last one writes the results.
    float* acc = a.ws + ((int64_t)slot * a.Hv + hk * gr) * ws_tile(DK, DV) + ws_S(DV) + 4 * tid;
    float end = 0.f;
    T* const dQp = (T*)a.dQ + kat;
    T* const dKp = (T*)a.dK + kat;
#pragma unroll
    for (int i = 0; i < NR; ++i) {
      // row form: this lane has row r, 4 columns
      const int I = I0 + i, r = 16 * I + c;
      const float bt = sr[0][r], eg = sr[1][r], er = sr[2][r];
      f32x4 F_[2], km[2], ke[2], R[2], kv[2], qv[2];
#pragma unroll
      for (int b = 0; b < 2; ++b) {
        kv[b] = load4(sm + G::oK + r * LDK + col + 16 * b + 4 * g);
        qv[b] = load4(sm + G::oQ + r * LDK + col + 16 * b + 4 * g);
        dq[b][i] *= eg * a.scale;
        R[b] = km[b] = er * yd[b][i];
        F_[b] = ke[b] = zero4();
      }
#pragma unroll
      for (int p = 0; p < 2; ++p) {
        if (p <= I / 2) {
          const Terms<F> P = load_terms<F>(sm + G::oPr, t_slot(I, p), l);
          const Terms<F> Er = load_terms<F>(sm + G::oEr, t_slot(I, p), l);
#pragma unroll
          for (int k = NT - 1; k >= 0; --k)
#pragma unroll
            for (int b = 0; b < 2; ++b) {
              dq[b][i] = Pair<F>::template mma<true>(P.t[k], kf[b][p], dq[b][i]);
              F_[b] = Pair<F>::template mma<true>(Er.t[k], kf[b][p], F_[b]);
            }
        }
        if (p >= I / 2) {
          const Terms<F> P = load_terms<F>(sm + G::oPc, tt_slot(I, p), l);
          const Terms<F> Ec = load_terms<F>(sm + G::oEc, tt_slot(I, p), l);
#pragma unroll
          for (int k = NT - 1; k >= 0; --k)
#pragma unroll
            for (int b = 0; b < 2; ++b) {
              km[b] = Pair<F>::template mma<true>(P.t[k], qf[b][p], km[b]);
              ke[b] = Pair<F>::template mma<true>(Ec.t[k], kf[b][p], ke[b]);
            }
        }
      }
      float dotF = 0.f, dotG = 0.f;
#pragma unroll
      for (int b = 0; b < 2; ++b) {
        const f32x4 kp = bt * (F_[b] - eg * zs[b][i]);
        km[b] += ke[b];
#pragma unroll
        for (int v = 0; v < 4; ++v) {
          dotF = __builtin_fmaf(kv[b][v], F_[b][v], dotF);
          dotG += qv[b][v] * dq[b][i][v] + kv[b][v] * (kp[v] - km[b][v]);
          end = __builtin_fmaf(kv[b][v], R[b][v], end);
        }
        f32x4 sq = dq[b][i], sk = kp + km[b];
        float* at = acc + (b * NR + i) * 2 * 2048;
        if (h > hk * gr) {
          sq += at4(at);
          sk += at4(at + 2048);
        }
        if (h + 1 < (hk + 1) * gr) {
          *(f32x4*)at = sq;
          *(f32x4*)(at + 2048) = sk;
        } else if (r < m) {
          const uint32_t to = (uint32_t)r * (uint32_t)kld + (uint32_t)(col + 16 * b + 4 * g);
          store4(dQp + to, sq);
          store4(dKp + to, sk);
        }
      }
      dotF = sum_apart32(sum_apart16(dotF));
      dotG = sum_apart32(sum_apart16(dotG));
      if (g == 0) {
        red[0][wv % G::NC][r] = dotF;
        red[1][wv % G::NC][r] = dotG;
      }
    }
    // (every row group has formed the same <S, dS> of its columns)
    if (I0 == 0) end = __builtin_fmaf(sr[1][BC - 1], ss, end);
    end = sum_lanes<64>(end);
    if (l == 0) send[wv] = end;
    __syncthreads();
    if (tid < BC) {
      const int r = tid;
      float db = 0.f, dg = 0.f;
#pragma unroll
      for (int i = 0; i < NJ; ++i) db += sdb[i][r];
#pragma unroll
      for (int i = 0; i < G::NC; ++i) {
        db += red[0][i][r];
        dg += red[1][i][r];
      }
      if (r == m - 1)
        dg += ((send[0] + send[1]) + (send[2] + send[3])) +
              ((send[4] + send[5]) + (send[6] + send[7]));
      sdg[r] = dg;
      if (r < m) a.dbeta[(t0 + r) * a.Hv + h] = db;
    }
    __syncthreads();
    if (tid < m) a.dg[(t0 + tid) * a.Hv + h] = part_sum(sdg, tid, m, a.C);
  }
}

// The same with four waves and half the LDS, for more chunks than CUs: two workgroups
// share a CU, each in its own phase, so that one's matrix work runs beside the other's
// vector work and loads.  The value columns are taken 64 at a time; P and E take the
// place of what they were formed from one after the other.  The states' terms are those
// of S, then those of dS: both at once, or the next pair's states asked for ahead, went
// to scratch (168 us became 185 and more).
// Bound: vector instructions (37% of the cycles), matrix instructions (27%), LDS (28%) of
// two waves a SIMD, and their waits for memory.  8192 tokens of 16 heads of 128 by 128 in
// bf16 take 173 us, 300 KB a chunk and head at 3.6 TB/s; 4 x 8192 of 32 value heads 1.33 ms,
// 4.3 TB/s (42, 31 and 31%).
template <int DK, int DV>
struct Halves {
  static constexpr int NC = DK / 32, RG = 4 / NC, NR = 4 / RG, LDK = DK + 8;
  // LDS, in bf16 values: T, and dO, dZ and Y of 64 value columns; later P or E along its
  // rows and down them, the rows of K and Q, and a block a wave to transpose by
  static constexpr int oT = 0, oO = 18 * 512, oZ = oO + 8 * 512, oY = oZ + 24 * 512;
  static constexpr int oEnd = oY + 24 * 512;
  static constexpr int oR = 0, oC = 18 * 512, oK = 36 * 512, oQ = oK + BC * LDK;
  static constexpr int oTr = oQ + BC * LDK, oEnd2 = oTr + 4 * 512;
  static constexpr int SIZE = oEnd2 > oEnd ? oEnd2 : oEnd;
};

template <int DK, int DV>
__global__ __launch_bounds__(256, 2) void k_bwd_grads_half(const BwdArgs a) {
  typedef Halves<DK, DV> G;
  typedef __bf16 T;
  typedef bf16x4 F;
  typedef bf16x8 Vec;
  constexpr int NR = G::NR, LDK = G::LDK, NJ = DV / 16;
  __shared__ __attribute__((aligned(16))) T sm[G::SIZE];
  __shared__ __attribute__((aligned(16))) float sr[5][BC];
  __shared__ float sdb[NJ][BC], red[2][G::NC][BC], sdg[BC], send[4];
  const uint32_t slot = blockIdx.x / (uint32_t)a.Hk;
  const int hk = (int)(blockIdx.x - slot * (uint32_t)a.Hk), gr = a.gr;
  int64_t t0 = 0;
  const int m = chunk_at(a, slot, t0);
  if (m == 0) return;
  const int wv = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int col = 32 * (wv % G::NC), I0 = G::RG == 1 ? 0 : wv / G::NC * NR;
  const int64_t kat = (t0 * a.Hk + hk) * DK;
  const uint32_t kld = (uint32_t)a.Hk * DK, vld = (uint32_t)a.Hv * DV;

  for (int h = hk * gr; h < (hk + 1) * gr; ++h) {
    int tid = threadIdx.x;  // (a value of its own in every turn, as above)
    asm volatile("" : "+v"(tid));
    const Lane ln{tid & 63};
    const int l = ln.id, g = ln.g(), c = ln.c();
    float* ws = a.ws + ((int64_t)slot * a.Hv + h) * ws_tile(DK, DV);
    // a 16 x 16 block from column form to row form: row 4g + v lies at 4v + g
    auto turn_in = [&](float* t, const f32x4& x) __attribute__((always_inline)) {
#pragma unroll
      for (int v = 0; v < 4; ++v) t[(4 * v + g) * 16 + c] = x[v];
    };
    auto turn_out = [&](const float* t) __attribute__((always_inline)) {
      return at4(t + (4 * (c & 3) + (c >> 2)) * 16 + 4 * g);
    };
    // the blocks of dP (kind 0) and E (1) of this wave: an E costs as much as two of dP
    struct Blk {
      int kind, I, J;
    };
    Blk bk[5];
#pragma unroll
    for (int i = 0; i < 5; ++i) {
      const int e = wv < 2 ? 3 : 2;  // this wave's blocks of E come first
      const int n = wv < 2 ? (i < 3 ? 3 * wv + i : 2 * wv + i - 3)
                           : (i < 2 ? 2 + 2 * wv + i : 3 * wv + i - 4);
      const int I = n < 1 ? 0 : n < 3 ? 1 : n < 6 ? 2 : 3;
      bk[i] = Blk{i < e, I, n - I * (I + 1) / 2};
    }
    f32x4 pe[5], dq[2][NR], zs[2][NR], yd[2][NR];
    float ss = 0.f;
#pragma unroll
    for (int i = 0; i < 5; ++i) pe[i] = zero4();
#pragma unroll
    for (int b = 0; b < 2; ++b)
#pragma unroll
      for (int i = 0; i < NR; ++i) dq[b][i] = zs[b][i] = yd[b][i] = zero4();

#pragma unroll 1
    for (int vh = 0; vh < DV / 64; ++vh) {
      const int J = 4 * vh + wv;
      if (vh) __syncthreads();  // the last columns' operands have been used
      Terms<F> z[2];
      {
        f32x4 xb[4], zb[4], bt[4];
#pragma unroll
        for (int I = 0; I < 4; ++I) {
          xb[I] = at4(ws + ws_X(DV) + blk_at(I, J, NJ) + 4 * l);
          zb[I] = at4(ws + ws_R() + blk_at(I, J, NJ) + 4 * l);
          bt[I] = at4(ws + ws_rows() + 16 * I + 4 * g);
        }
        const T* dO = (const T*)a.dO + (t0 * a.Hv + h) * DV + 64 * vh;
        F o[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const int at = tid + 256 * i;
          o[i] = *(const F*)(dO + ((uint32_t)min(at >> 4, m - 1) * vld + (uint32_t)(4 * (at & 15))));
        }
        if (vh == 0) {
#pragma unroll
          for (int i = 0; i < 5; ++i) {
            const int at = tid + 256 * i, sl = at / 192;  // 192 pieces of 16 bytes a slot
            if (at < 6 * 192)
              *(Vec*)(sm + G::oT + at * 8) =
                  *(const Vec*)((const T*)(ws + ws_T() + TS * sl) + (at - 192 * sl) * 8);
          }
          for (int i = tid; i < 5 * BC; i += 256) (&sr[0][0])[i] = ws[ws_rows() + i];
        }
#pragma unroll
        for (int p = 0; p < 2; ++p)
          z[p] = split<F>(bt[2 * p] * xb[2 * p], bt[2 * p + 1] * xb[2 * p + 1]);
        float* t = (float*)(sm + G::oY) + 1024 * wv;  // (Y is not there yet)
#pragma unroll
        for (int I = 0; I < 4; ++I) {
          turn_in(t + 256 * I, zb[I]);
#pragma unroll
          for (int v = 0; v < 4; ++v) {
            const float d = sum16(xb[I][v] * zb[I][v]);
            if (c == 0) sdb[J][16 * I + 4 * g + v] = d;
          }
        }
        lds_sync<true>();
#pragma unroll
        for (int I = 0; I < 4; ++I)
          store_half<F>(sm + G::oZ, 2 * I + (wv >> 1), wv & 1,
                        split_half<F>(turn_out(t + 256 * I)), l);
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const int at = tid + 256 * i, r = at >> 4, e = at & 15;
          *(F*)(sm + G::oO + ((r >> 4) * 2 + (e >> 3)) * 512 + 8 * (16 * (e & 3) + (r & 15)) +
                4 * ((e >> 2) & 1)) = r < m ? o[i] : F{};
        }
      }
      __syncthreads();
      // ---- Y = T Z, column block J
      {
        f32x4 y[4], yl[4];
#pragma unroll
        for (int I = 0; I < 4; ++I) y[I] = yl[I] = zero4();
#pragma unroll
        for (int p = 0; p < 2; ++p)
#pragma unroll
          for (int I = 2 * p; I < 4; ++I)
            mma_both<true>(load_terms<F>(sm + G::oT, t_slot(I, p), l), z[p], y[I], yl[I]);
#pragma unroll
        for (int I = 0; I < 4; ++I)
          store_half<F>(sm + G::oY, 2 * I + (wv >> 1), wv & 1, split_half<F>(y[I] + yl[I]), l);
      }
      __syncthreads();
#pragma unroll 1
      for (int p = 0; p < 2; ++p) {
        // S and dS, then dP and E while they are on their way
        const int at = blk_at(col / 16, 4 * vh + 2 * p, NJ) + 4 * l;
        const float *S = ws + ws_S(DV) + at, *dS = ws + ws_dS(DK, DV) + at;
        f32x4 s_[2][2], d_[2][2];
#pragma unroll
        for (int b = 0; b < 2; ++b)
#pragma unroll
          for (int hf = 0; hf < 2; ++hf) {
            s_[b][hf] = at4(S + blk_at(b, hf, NJ));
            d_[b][hf] = at4(dS + blk_at(b, hf, NJ));
          }
#pragma unroll
        for (int i = 0; i < 5; ++i) {
          const Terms<F> y = load_terms<F>(sm + G::oY, 2 * bk[i].J + p, l);
          const int at = 2 * bk[i].I + p;
          if (i < 2 || (i == 2 && wv < 2)) {
            f32x4 low = zero4();
            mma_both<false>(load_terms<F>(sm + G::oZ, at, l), y, pe[i], low);
            pe[i] += low;
          } else {
            pe[i] = mma_in<false>(slot_load<F>(sm + G::oO + at * 512, l), y, pe[i]);
          }
        }
        // ---- dO S^T, dZ S^T, Y dS^T and <S, dS>; one state's terms at a time
        constexpr int tx[6] = {0, 1, 2, 1, 0, 0}, ty[6] = {2, 1, 0, 0, 1, 0};
#pragma unroll
        for (int b = 0; b < 2; ++b)
#pragma unroll
          for (int hf = 0; hf < 2; ++hf)
#pragma unroll
            for (int v = 0; v < 4; ++v) ss = __builtin_fmaf(s_[b][hf][v], d_[b][hf][v], ss);
        {
          const Terms<F> sv[2] = {split<F>(s_[0][0], s_[0][1]), split<F>(s_[1][0], s_[1][1])};
#pragma unroll
          for (int i = 0; i < NR; ++i) {
            const int at = 2 * (I0 + i) + p;
            const Pair<F> o = slot_load<F>(sm + G::oO + at * 512, l);
            const Terms<F> z = load_terms<F>(sm + G::oZ, at, l);
#pragma unroll
            for (int k = 0; k < 6; ++k)
#pragma unroll
              for (int b = 0; b < 2; ++b) {
                zs[b][i] = Pair<F>::template mma<true>(z.t[tx[k]], sv[b].t[ty[k]], zs[b][i]);
                if (k >= 3) dq[b][i] = Pair<F>::template mma<true>(o, sv[b].t[5 - k], dq[b][i]);
              }
          }
        }
        {
          const Terms<F> dv[2] = {split<F>(d_[0][0], d_[0][1]), split<F>(d_[1][0], d_[1][1])};
#pragma unroll
          for (int i = 0; i < NR; ++i) {
            const Terms<F> y = load_terms<F>(sm + G::oY, 2 * (I0 + i) + p, l);
#pragma unroll
            for (int k = 0; k < 6; ++k)
#pragma unroll
              for (int b = 0; b < 2; ++b)
                yd[b][i] = Pair<F>::template mma<true>(y.t[tx[k]], dv[b].t[ty[k]], yd[b][i]);
          }
        }
      }
    }
#pragma unroll
    for (int i = 0; i < 5; ++i) {
      const int r0 = 16 * bk[i].I + 4 * g, j = 16 * bk[i].J + c;
      const float s = bk[i].kind ? -1.f : a.scale;
      const int lo = bk[i].kind ? j + 1 : j;  // the first row that has this column
#pragma unroll
      for (int v = 0; v < 4; ++v) {
        const float d = __expf((sr[3][r0 + v] - sr[3][j]) + (sr[4][r0 + v] - sr[4][j]));
        pe[i][v] = r0 + v >= lo ? s * d * pe[i][v] : 0.f;
      }
    }
    constexpr int CPR = DK / 8, KN = BC * CPR / 256;
    Vec kv[KN], qv[KN];
#pragma unroll
    for (int i = 0; i < KN; ++i) {
      const int at = tid + 256 * i;
      const uint32_t from = (uint32_t)min(at / CPR, m - 1) * kld + (uint32_t)(at % CPR * 8);
      kv[i] = *(const Vec*)((const T*)a.K + kat + from);
      qv[i] = *(const Vec*)((const T*)a.Q + kat + from);
    }
    // the blocks of one kind as left operands: along their rows, and down them (E with beta)
    auto lay = [&](int kind) __attribute__((always_inline)) {
      float* t = (float*)(sm + G::oTr) + 256 * wv;
#pragma unroll
      for (int i = 0; i < 5; ++i) {
        if (bk[i].kind != kind) continue;
        const int I = bk[i].I, J = bk[i].J;
        turn_in(t, pe[i]);
        lds_sync<true>();
        store_half<F>(sm + G::oR, t_slot(I, J >> 1), J & 1, split_half<F>(turn_out(t)), l);
        lds_sync<true>();
        store_half<F>(sm + G::oC, tt_slot(J, I >> 1), I & 1,
                      split_half<F>(kind ? at4(&sr[0][16 * I + 4 * g]) * pe[i] : pe[i]), l);
        if (I == J) {  // the block beside the diagonal that its pair takes along: zeros
          if (I % 2 == 0)
            store_half<F>(sm + G::oR, t_slot(I, I >> 1), 1, split_half<F>(zero4()), l);
          else
            store_half<F>(sm + G::oC, tt_slot(I, I >> 1), 0, split_half<F>(zero4()), l);
        }
      }
    };
    __syncthreads();
#pragma unroll
    for (int i = 0; i < KN; ++i) {
      const int at = tid + 256 * i, r = at / CPR, e = at % CPR * 8;
      *(Vec*)(sm + G::oK + r * LDK + e) = r < m ? kv[i] : Vec{};
      *(Vec*)(sm + G::oQ + r * LDK + e) = r < m ? qv[i] : Vec{};
    }
    lay(0);
    __syncthreads();
    // ---- dP K and dP^T Q; then E K and E^T beta K
    Pair<F> kf[2][2];
    float end = 0.f;
    {
      Pair<F> qf[2][2];
#pragma unroll
      for (int b = 0; b < 2; ++b)
#pragma unroll
        for (int p = 0; p < 2; ++p) {
          kf[b][p] = col_pair<LDK>(sm + G::oK, 32 * p, col + 16 * b, ln);
          qf[b][p] = col_pair<LDK>(sm + G::oQ, 32 * p, col + 16 * b, ln);
        }
#pragma unroll
      for (int i = 0; i < NR; ++i) {
        const int I = I0 + i, r = 16 * I + c;
        const float eg = sr[1][r] * a.scale, er = sr[2][r];
#pragma unroll
        for (int b = 0; b < 2; ++b) {
          const f32x4 k = load4(sm + G::oK + r * LDK + col + 16 * b + 4 * g);
          dq[b][i] *= eg;
          yd[b][i] *= er;
#pragma unroll
          for (int v = 0; v < 4; ++v) end = __builtin_fmaf(k[v], yd[b][i][v], end);
        }
#pragma unroll
        for (int p = 0; p < 2; ++p) {
          if (p <= I / 2) {
            const Terms<F> P = load_terms<F>(sm + G::oR, t_slot(I, p), l);
#pragma unroll
            for (int t = 2; t >= 0; --t)
#pragma unroll
              for (int b = 0; b < 2; ++b)
                dq[b][i] = Pair<F>::template mma<true>(P.t[t], kf[b][p], dq[b][i]);
          }
          if (p >= I / 2) {
            const Terms<F> P = load_terms<F>(sm + G::oC, tt_slot(I, p), l);
#pragma unroll
            for (int t = 2; t >= 0; --t)
#pragma unroll
              for (int b = 0; b < 2; ++b)
                yd[b][i] = Pair<F>::template mma<true>(P.t[t], qf[b][p], yd[b][i]);
          }
        }
      }
    }
    __syncthreads();
    lay(1);
    __syncthreads();
    // The sums over the value heads of a key head, as above.
    float* acc = a.ws + ((int64_t)slot * a.Hv + hk * gr) * ws_tile(DK, DV) + ws_S(DV) + 4 * tid;
    T* const dQp = (T*)a.dQ + kat;
    T* const dKp = (T*)a.dK + kat;
#pragma unroll
    for (int i = 0; i < NR; ++i) {
      const int I = I0 + i, r = 16 * I + c;
      const float bt = sr[0][r], eg = sr[1][r];
      f32x4 F_[2] = {zero4(), zero4()};
#pragma unroll
      for (int p = 0; p < 2; ++p) {
        if (p <= I / 2) {
          const Terms<F> Er = load_terms<F>(sm + G::oR, t_slot(I, p), l);
#pragma unroll
          for (int t = 2; t >= 0; --t)
#pragma unroll
            for (int b = 0; b < 2; ++b)
              F_[b] = Pair<F>::template mma<true>(Er.t[t], kf[b][p], F_[b]);
        }
        if (p >= I / 2) {
          const Terms<F> Ec = load_terms<F>(sm + G::oC, tt_slot(I, p), l);
#pragma unroll
          for (int t = 2; t >= 0; --t)
#pragma unroll
            for (int b = 0; b < 2; ++b)
              yd[b][i] = Pair<F>::template mma<true>(Ec.t[t], kf[b][p], yd[b][i]);
        }
      }
      float dotF = 0.f, dotG = 0.f;
#pragma unroll
      for (int b = 0; b < 2; ++b) {
        const f32x4 k = load4(sm + G::oK + r * LDK + col + 16 * b + 4 * g);
        const f32x4 q = load4(sm + G::oQ + r * LDK + col + 16 * b + 4 * g);
        const f32x4 kp = bt * (F_[b] - eg * zs[b][i]);
#pragma unroll
        for (int v = 0; v < 4; ++v) {
          dotF = __builtin_fmaf(k[v], F_[b][v], dotF);
          dotG += q[v] * dq[b][i][v] + k[v] * (kp[v] - yd[b][i][v]);
        }
        f32x4 sq = dq[b][i], sk = kp + yd[b][i];
        float* at = acc + (b * NR + i) * 2 * 1024;
        if (h > hk * gr) {
          sq += at4(at);
          sk += at4(at + 1024);
        }
        if (h + 1 < (hk + 1) * gr) {
          *(f32x4*)at = sq;
          *(f32x4*)(at + 1024) = sk;
        } else if (r < m) {
          const uint32_t to = (uint32_t)r * kld + (uint32_t)(col + 16 * b + 4 * g);
          store4(dQp + to, sq);
          store4(dKp + to, sk);
        }
      }
      dotF = sum_apart32(sum_apart16(dotF));
      dotG = sum_apart32(sum_apart16(dotG));
      if (g == 0) {
        red[0][wv % G::NC][r] = dotF;
        red[1][wv % G::NC][r] = dotG;
      }
    }
    // (every row group has formed the same <S, dS> of its columns)
    if (I0 == 0) end = __builtin_fmaf(sr[1][BC - 1], ss, end);
    end = sum_lanes<64>(end);
    if (l == 0) send[wv] = end;
    __syncthreads();
    if (tid < BC) {
      const int r = tid;
      float db = 0.f, dg = 0.f;
#pragma unroll
      for (int i = 0; i < NJ; ++i) db += sdb[i][r];
#pragma unroll
      for (int i = 0; i < G::NC; ++i) {
        db += red[0][i][r];
        dg += red[1][i][r];
      }
      if (r == m - 1) dg += (send[0] + send[1]) + (send[2] + send[3]);
      sdg[r] = dg;
      if (r < m) a.dbeta[(t0 + r) * a.Hv + h] = db;
    }
    __syncthreads();
    if (tid < m) a.dg[(t0 + tid) * a.Hv + h] = part_sum(sdg, tid, m, a.C);
  }
}

int64_t backward_slots(int nseq, int L, bool packed) {
  return packed ? (int64_t)L / BC + nseq : nseq * (((int64_t)L + BC - 1) / BC);
}
int64_t backward_tile_bytes(int dk, int dv) { return ws_tile(dk, dv) * 4; }

template <int DK, int DV, typename T>
static hipError_t run_backward(const BwdArgs& a, int64_t slots, hipStream_t st) {
  if (slots > 0)
    hipLaunchKernelGGL((k_bwd_prep<DK, DV, T>), dim3((unsigned)(slots * a.Hv)), dim3(256), 0, st, a);
  if (slots > 0 || a.dS0) {
    const hipError_t e = launch_walks(a, DK, DV, sizeof(T) == 4 ? 0 : 1, st);
    if (e != hipSuccess) return e;
  }
  if (slots > 0) {
    const unsigned tiles = (unsigned)(slots * a.Hk);
    if constexpr (sizeof(T) == 2) {
      // With no CU left over, two workgroups of four waves a CU; until then one of eight,
      // which has a chunk done sooner: us of the two for DK = DV = 128, 64 chunks by key
      // heads 24.6 and 19.5, 256 30.1 and 25.7, 320 37.7 and 43.1, 1024 83 and 101; 1024
      // of 64 by 64 47 and 56.
      if (tiles > 256) {
        hipLaunchKernelGGL((k_bwd_grads_half<DK, DV>), dim3(tiles), dim3(256), 0, st, a);
        return hipGetLastError();
      }
    }
    hipLaunchKernelGGL((k_bwd_grads<DK, DV, T>), dim3(tiles), dim3(512), 0, st, a);
  }
  return hipGetLastError();
}

hipError_t launch_backward(const void* Q, const void* K, const void* V, const float* beta,
                           const float* g, const void* dO, const float* S0, const float* dSf,
                           void* dQ, void* dK, void* dV, float* dbeta, float* dg, float* dS0,
                           float* ws, const int* cu, int nseq, int L, int Hk, int Hv, int dk,
                           int dv, int C, float scale, int dtype, hipStream_t st) {
  BwdArgs a{Q,  K,     V,  dO,  beta, g,  S0,   dSf, dQ,              dK, dV, dbeta,
            dg, dS0,   ws, cu,  nseq, L,  (L + BC - 1) / BC, Hk, Hv, C, scale, Hk ? Hv / Hk : 1};
  const int64_t slots = L > 0 ? backward_slots(nseq, L, cu != nullptr) : 0;
  GDN_DK_SWITCH(dk, GDN_DV_SWITCH(dv, {
    return dtype == 0 ? run_backward<DK, DV, float>(a, slots, st)
                      : run_backward<DK, DV, __bf16>(a, slots, st);
  }))
  return hipErrorNotSupported;
}

}  // namespace gdn
