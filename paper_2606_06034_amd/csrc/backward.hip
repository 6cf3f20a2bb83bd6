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
// Four launches: k_bwd_prep (every chunk: T, P^T dO), k_bwd_states (the states
// entering the chunks, first to last), k_bwd_reverse (the gradients of the
// states leaving them, last to first), k_bwd_grads (every chunk: the
// gradients).  The chunks here are always of 64 tokens, whatever chunk size
// the caller's g restarts at (16, 32 or 64): the result of the exact layer
// does not depend on it, and gamma is g plus the last g of the 64-chunk's
// earlier parts.
//
// Everything is formed in fp32, bf16 inputs too: the gradients of beta and g
// are differences of large sums, and their outputs are fp32.
#include "chunk.hpp"
#include "engine.hpp"
#include "launch.hpp"
#include "layer.hpp"
#include "split.hpp"

namespace gdn {

namespace {

constexpr int BC = 64;  // tokens a chunk

// Workspace of one (chunk, value head), in floats.  T and T^T lie as the terms
// (split.hpp) of the pair fragments of their row blocks, 3 KB a fragment (2 KB
// with fp32 inputs): T (I, p) with 2p <= I, T^T (I, p) with 2p + 1 >= I.
constexpr int TS = 768;
__host__ __device__ constexpr int t_slot(int I, int p) { return (I == 3 ? 4 : I) + p; }
__host__ __device__ constexpr int tt_slot(int I, int p) { return (I < 2 ? 2 * I : 2 + I) + p - I / 2; }
__host__ __device__ constexpr int64_t ws_T() { return 0; }
__host__ __device__ constexpr int64_t ws_Tt() { return 6 * TS; }
__host__ __device__ constexpr int64_t ws_rows() { return 12 * TS; }  // beta e^g e^{gl-g} g off
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
__device__ __forceinline__ int chunk_at(const BwdArgs& a, int64_t slot, int64_t& t0) {
  int s;
  if (a.cu) {
    int lo = 0, hi = a.nseq;  // the last s with base(s) <= slot
    while (hi - lo > 1) {
      const int mid = (lo + hi) >> 1;
      if (a.cu[mid] / BC + mid <= slot) lo = mid; else hi = mid;
    }
    s = lo;
  } else {
    s = (int)(slot / a.nc);
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

// rows of [tokens, H, D] (row stride ld values) into LDS as fp32, rows of PD
// values; zeros past row m
template <int D, int PD, typename T>
__device__ __forceinline__ void rows_to_lds(float* s, const T* __restrict__ x, int64_t ld, int m) {
  constexpr int E = 16 / sizeof(T), CPR = D / E;
#pragma unroll
  for (int i = 0; i < BC * CPR / 256; ++i) {
    const int p = threadIdx.x + 256 * i, r = p / CPR, c = p % CPR * E;
    f32x4 v[E / 4];
#pragma unroll
    for (int k = 0; k < E / 4; ++k) v[k] = zero4();
    if (r < m)
#pragma unroll
      for (int k = 0; k < E / 4; ++k) v[k] = load4(x + r * ld + c + 4 * k);
#pragma unroll
    for (int k = 0; k < E / 4; ++k) *(f32x4*)(s + r * PD + c + 4 * k) = v[k];
  }
}

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

// one block of a pair's terms as values
__device__ __forceinline__ f32x4 half_of(const Terms<f32x4>& x, int hf) {
  return hf ? x.t[0].hi() : x.t[0].lo();
}
__device__ __forceinline__ f32x4 half_of(const Terms<bf16x4>& x, int hf) {
  return hf ? x.t[0].hi() + (x.t[1].hi() + x.t[2].hi()) : x.t[0].lo() + (x.t[1].lo() + x.t[2].lo());
}

template <typename T> struct FragOf { typedef f32x4 type; };
template <> struct FragOf<__bf16> { typedef bf16x4 type; };

}  // namespace

// ---- every chunk: T, T^T and P^T dO
template <int DK, int DV, typename T>
__global__ __launch_bounds__(256) void k_bwd_prep(const BwdArgs a) {
  typedef typename FragOf<T>::type F;
  constexpr int LD = BC + 4;
  __shared__ float sA[BC * LD], sP[BC * LD], sr[5][BC];
  const int64_t slot = blockIdx.x / a.Hv;
  const int h = (int)(blockIdx.x - slot * a.Hv), hk = h / (a.Hv / a.Hk);
  int64_t t0 = 0;
  const int m = chunk_at(a, slot, t0);
  if (m == 0) return;
  float* ws = a.ws + (int64_t)blockIdx.x * ws_tile(DK, DV);
  const int wv = threadIdx.x >> 6, g = lane_g(), c = lane_c();
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
  __syncthreads();
  // row block wv of A and P
  {
    Pair<F> q[DK / 32], k[DK / 32], kj[DK / 32];
    const int64_t ld = (int64_t)a.Hk * DK;
    const T* Kp = (const T*)a.K + (t0 * a.Hk + hk) * DK;
    const T* Qp = (const T*)a.Q + (t0 * a.Hk + hk) * DK;
    auto rows = [&](Pair<F>(&x)[DK / 32], const T* p, int I) __attribute__((always_inline)) {
      const int r = 16 * I + c, rr = r < m ? r : m - 1;
#pragma unroll
      for (int s = 0; s < DK / 32; ++s) {
        x[s] = load_row8<F>(p + rr * ld + 32 * s + 8 * g);
        if (r >= m) x[s] = Pair<F>::zero();
      }
    };
    rows(q, Qp, wv);
    rows(k, Kp, wv);
    for (int J = 0; J <= wv; ++J) {
      rows(kj, Kp, J);
      f32x4 kk = zero4(), qk = zero4();
#pragma unroll
      for (int s = 0; s < DK / 32; ++s) {
        kk = Pair<F>::template mma<false>(k[s], kj[s], kk);
        qk = Pair<F>::template mma<false>(q[s], kj[s], qk);
      }
#pragma unroll
      for (int v = 0; v < 4; ++v) {
        const int i = 16 * wv + 4 * g + v, j = 16 * J + c;
        const float d = i >= j ? expf((sr[3][i] - sr[3][j]) + (sr[4][i] - sr[4][j])) : 0.f;
        sA[i * LD + j] = i > j ? -sr[0][i] * kk[v] * d : 0.f;
        sP[i * LD + j] = i >= j ? a.scale * qk[v] * d : 0.f;
      }
    }
  }
  __syncthreads();
  if (wv == 0) {
    Acc<4> Lr, Tr;
#pragma unroll
    for (int I = 0; I < 4; ++I)
#pragma unroll
      for (int J = 0; J <= I; ++J)
        Lr.a[bidx(I, J)] = at4(sA + (16 * I + c) * LD + 16 * J + 4 * g);
    blockwise_inverse<4, f32x4>(Lr, Tr);
    const f32x4 z = zero4();
#pragma unroll
    for (int I = 0; I < 4; ++I)
#pragma unroll
      for (int J = 0; J < 4; ++J) {
        // (sA holds nothing that another wave reads)
        if (J <= I) *(f32x4*)(sA + (16 * I + c) * LD + 16 * J + 4 * g) = Tr.a[bidx(I, J)];
        if (J / 2 <= I / 2)
          store_half<F>((T*)(ws + ws_T() + TS * t_slot(I, J / 2)), 0, J & 1,
                        split_half<F>(J <= I ? Tr.a[bidx(I, J)] : z), lane_id());
      }
    lds_sync<true>();
#pragma unroll
    for (int I = 0; I < 4; ++I)
#pragma unroll
      for (int J = 0; J < 4; ++J)
        if (J / 2 >= I / 2)
          store_half<F>(
              (T*)(ws + ws_Tt() + TS * tt_slot(I, J / 2)), 0, J & 1,
              split_half<F>(J >= I ? down4(sA + (16 * J + 4 * g) * LD + 16 * I + c, LD) : z),
              lane_id());
  } else {
    const T* dO = (const T*)a.dO + (t0 * a.Hv + h) * DV;
    for (int J = wv - 1; J < DV / 16; J += 3) {
      f32x4 o[4];
#pragma unroll
      for (int k = 0; k < 4; ++k) o[k] = col_block(dO + 16 * J, (int64_t)a.Hv * DV, 16 * k, m);
#pragma unroll
      for (int I = 0; I < 4; ++I) {
        f32x4 x = zero4();
#pragma unroll
        for (int k = I; k < 4; ++k)
          x = mma16(down4(sP + (16 * k + 4 * g) * LD + 16 * I + c, LD), o[k], x);
#pragma unroll
        for (int v = 0; v < 4; ++v) ws[ws_R() + (16 * I + 4 * g + v) * DV + 16 * J + c] = x[v];
      }
    }
  }
}

// A walk over the chunks of one (sequence, value head) for 16 value columns, four
// waves.  The [dk, 16] part of the state lies in registers, wave w holding its
// rows 32w .. 32w + 31 (two blocks, one pair).  A step is serial, so the
// waves share each of its products: a product with the state is summed over
// the waves' own rows (no wave needs another's state), the sums, then Z (dY)
// and Y (dX) of row block w go through LDS, three exchanges a chunk.
template <int DK, int DV, typename T>
struct Walk {
  typedef typename FragOf<T>::type F;
  static constexpr int NT = TermsOf<F>::N, NQ = DK / 32, NS = DV / 16;
  static constexpr int E = 16 / sizeof(T), LD = DK + E;  // rows in LDS, 16 bytes apart
  static constexpr int CPR = DK / E, KI = BC * CPR / 256;
  typedef T Vec __attribute__((ext_vector_type(E)));
  // (sequence, value head) and first value column of this workgroup.  Workgroups
  // are dealt to the 8 XCDs in turn; all slices of a head go to one XCD, whose
  // L2 then reads the head's chunks once.
  static __device__ __forceinline__ int64_t head_of(int& n0) {
    const unsigned x = blockIdx.x, r = x >> 3;
    n0 = (int)(r % NS) * 16;
    return (int64_t)(r / NS) * 8 + (x & 7);
  }
  // A chunk's rows of K (Q) on their way to LDS.  Byte offsets from the chunk's
  // first row: at most 64 rows of all heads, 32 bits; those of the rows past
  // the chunk's last are clamped to it by their size.
  struct Rows {
    Vec v[KI];
  };
  static __device__ __forceinline__ void fetch(Rows& x, const T* p, const uint32_t (&off)[KI],
                                               uint32_t last) {
    const uint32_t col = threadIdx.x % CPR * 16;
#pragma unroll
    for (int i = 0; i < KI; ++i)
      x.v[i] = *(const Vec*)((const char*)p + (min(off[i], last) + col));
  }
  static __device__ __forceinline__ void put(T* s, const Rows& x, int m) {
    T* to = s + threadIdx.x / CPR * LD + threadIdx.x % CPR * E;
    if (m == BC) {
#pragma unroll
      for (int i = 0; i < KI; ++i) *(Vec*)(to + 256 / CPR * i * LD) = x.v[i];
    } else {
#pragma unroll
      for (int i = 0; i < KI; ++i)
        *(Vec*)(to + 256 / CPR * i * LD) =
            (int)threadIdx.x / CPR + 256 / CPR * i < m ? x.v[i] : Vec{};
    }
  }
  // row block w of T (or T^T): two pairs of terms at most
  struct TRow {
    Terms<F> v[2];
  };
  static __device__ __forceinline__ void fetch_t(TRow& x, const float* p, int n, int l) {
#pragma unroll
    for (int i = 0; i < 2; ++i)
      if (i < n) x.v[i] = load_terms<F>((const T*)(p + TS * i), 0, l);
  }
  // this wave's share of the product of the 64 rows in LDS with the state
  static __device__ __forceinline__ void share(const T* sK, const Terms<F>& s, float* part, int wv,
                                               Lane ln) {
#pragma unroll
    for (int I = 0; I < 4; ++I)
      *(f32x4*)(part + (4 * wv + I) * 256 + 4 * ln.id) =
          mma_in<false>(row_pair<LD>(sK, 16 * I, 32 * wv, ln), s, zero4());
  }
  // the sum of the shares of row block wv
  static __device__ __forceinline__ f32x4 sum(const float* part, int wv, int l) {
    f32x4 x[NQ];
#pragma unroll
    for (int q = 0; q < NQ; ++q) x[q] = at4(part + (4 * q + wv) * 256 + 4 * l);
    if constexpr (NQ == 4) return (x[0] + x[1]) + (x[2] + x[3]);
    return x[0] + x[1];
  }
  // the transposed rows of this wave's two state blocks: [block][token pair]
  struct Cols {
    Pair<F> v[2][2];
  };
  static __device__ __forceinline__ void cols(Cols& x, const T* s, int wv, Lane ln) {
#pragma unroll
    for (int h = 0; h < 2; ++h)
#pragma unroll
      for (int p = 0; p < 2; ++p) x.v[h][p] = col_pair<LD>(s, 32 * p, 32 * wv + 16 * h, ln);
  }
  static __device__ __forceinline__ void state_in(f32x4 (&st)[2], const float* p, int n0, int wv) {
#pragma unroll
    for (int h = 0; h < 2; ++h)
      st[h] = p && wv < NQ ? col_block(p + n0, DV, 32 * wv + 16 * h, DK) : zero4();
  }
  static __device__ __forceinline__ void state_out(float* p, const f32x4 (&st)[2], int n0, int wv) {
    const uint32_t at = (32 * wv + 4 * lane_g()) * DV + n0 + lane_c();
#pragma unroll
    for (int h = 0; h < 2; ++h)
#pragma unroll
      for (int v = 0; v < 4; ++v) p[at + (16 * h + v) * DV] = st[h][v];
  }
  // 4 rows from r0 of a [64, DV] array
  static __device__ __forceinline__ void rows_out(float* p, f32x4 x, int n0, int r0) {
    const uint32_t at = r0 * DV + n0 + lane_c();
#pragma unroll
    for (int v = 0; v < 4; ++v) p[at + v * DV] = x[v];
  }
  // this lane's rows 16 wv + 4g + v of a column of V (dO): byte offsets as above
  static __device__ __forceinline__ RawBlock<T> fetch_col(const T* p, const uint32_t (&off)[4],
                                                          uint32_t last) {
    RawBlock<T> x;
    const uint32_t col = lane_c() * sizeof(T);
#pragma unroll
    for (int v = 0; v < 4; ++v) x.v[v] = *(const T*)((const char*)p + (min(off[v], last) + col));
    return x;
  }
};

// ---- the states entering the chunks
template <int DK, int DV, typename T>
__global__ __launch_bounds__(256) void k_bwd_states(const BwdArgs a) {
  typedef Walk<DK, DV, T> W;
  typedef typename W::F F;
  __shared__ __attribute__((aligned(16))) T sK[BC * W::LD];
  __shared__ __attribute__((aligned(16))) float part[W::NQ * 4 * 256];
  __shared__ __attribute__((aligned(16))) T sZ[2 * W::NT * 512], sY[2 * W::NT * 512];
  int n0;
  const int64_t sh = W::head_of(n0);
  if (sh >= (int64_t)a.nseq * a.Hv) return;  // the whole workgroup, before any barrier
  const int s = (int)(sh / a.Hv);
  const int h = (int)(sh - (int64_t)s * a.Hv), hk = h / (a.Hv / a.Hk);
  const Seq sq(a, s);
  const int wv = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), nc = sq.chunks();
  const Lane ln = lane_here();
  const int l = ln.id, g = ln.g(), c = ln.c(), r0 = 16 * wv + 4 * g;
  const bool owner = wv < W::NQ;
  const int64_t kld = (int64_t)a.Hk * DK, vld = (int64_t)a.Hv * DV;
  uint32_t koff[W::KI], voff[4];  // byte offsets of this thread's rows of K, of V
#pragma unroll
  for (int i = 0; i < W::KI; ++i)
    koff[i] = (threadIdx.x + 256 * i) / W::CPR * (uint32_t)kld * sizeof(T);
#pragma unroll
  for (int v = 0; v < 4; ++v) voff[v] = (r0 + v) * (uint32_t)vld * sizeof(T);
  f32x4 st[2];
  W::state_in(st, a.S0 ? a.S0 + sh * DK * DV : nullptr, n0, wv);
  if (nc == 0) return;
  auto tile = [&](int ck) { return a.ws + ((sq.base + ck) * a.Hv + h) * ws_tile(DK, DV); };
  auto rows = [&](int ck) { return min(BC, sq.len - ck * BC); };
  // what a chunk needs besides K, asked for a chunk ahead
  struct Ops {
    RawBlock<T> v;
    f32x4 beta, eg, er;
    float el;
    typename W::TRow t;
  };
  auto fetch = [&](Ops& x, int ck) __attribute__((always_inline)) {
    const float* ws = tile(ck);
    const float* rv = ws + ws_rows();
    W::fetch_t(x.t, ws + ws_T() + TS * t_slot(wv, 0), wv / 2 + 1, l);
    x.v = W::fetch_col((const T*)a.V + ((sq.t0 + (int64_t)ck * BC) * a.Hv + h) * DV + n0, voff,
                       (rows(ck) - 1) * (uint32_t)vld * sizeof(T));
    x.beta = at4(rv + r0);
    x.eg = at4(rv + BC + r0);
    x.er = at4(rv + 2 * BC + r0);
    x.el = rv[2 * BC - 1];
  };
  auto keys = [&](typename W::Rows& x, int ck) __attribute__((always_inline)) {
    W::fetch(x, (const T*)a.K + ((sq.t0 + (int64_t)ck * BC) * a.Hk + hk) * DK, koff,
             (rows(ck) - 1) * (uint32_t)kld * sizeof(T));
  };
  const int last = nc - 1;
  // two sets, asked for two chunks ahead
  Ops ops[2];
  typename W::Rows krs[2];
  keys(krs[0], 0);
  fetch(ops[0], 0);
  W::put(sK, krs[0], rows(0));
  keys(krs[0], min(1, last));
  fetch(ops[1], min(1, last));
  keys(krs[1], min(2, last));
  lds_only_barrier();
  auto step = [&](int ck, Ops& op, typename W::Rows& kr) __attribute__((always_inline)) {
    float* ws = tile(ck);
    if (owner) {
      W::state_out(ws + ws_S(DV), st, n0, wv);
      W::share(sK, split<F>(st[0], st[1]), part, wv, ln);
    }
    lds_only_barrier();
    typename W::Cols kc;
    if (owner) W::cols(kc, sK, wv, ln);
    {
      const f32x4 x = block_of(op.v, 16 * wv, rows(ck)) - op.eg * W::sum(part, wv, l);
      W::rows_out(ws + ws_X(DV), x, n0, r0);
      store_half<F>(sZ, wv >> 1, wv & 1, split_half<F>(op.beta * x), l);
    }
    lds_only_barrier();
    W::put(sK, kr, rows(min(ck + 1, last)));
    keys(kr, min(ck + 3, last));
    __builtin_amdgcn_sched_barrier(0);
    {
      f32x4 y = zero4(), yl = zero4();
#pragma unroll
      for (int p = 0; p < 2; ++p)
        if (p <= wv / 2) mma_both<false>(op.t.v[p], load_terms<F>(sZ, p, l), y, yl);
      y += yl;
      store_half<F>(sY, wv >> 1, wv & 1, split_half<F>(op.er * y), l);
    }
    const float el = op.el;
    fetch(op, min(ck + 2, last));
    lds_only_barrier();
    if (owner) {
      f32x4 x[2] = {zero4(), zero4()};
#pragma unroll
      for (int p = 0; p < 2; ++p) {
        const Terms<F> y = load_terms<F>(sY, p, l);
#pragma unroll
        for (int hf = 0; hf < 2; ++hf) x[hf] = mma_in<false>(kc.v[hf][p], y, x[hf]);
      }
#pragma unroll
      for (int hf = 0; hf < 2; ++hf) st[hf] = st[hf] * el + x[hf];
    }
  };
  for (int ck = 0; ck < nc; ck += 2) {
    step(ck, ops[0], krs[0]);
    if (ck + 1 < nc) step(ck + 1, ops[1], krs[1]);
  }
}

// ---- the gradients of the states leaving the chunks, last chunk first
template <int DK, int DV, typename T>
__global__ __launch_bounds__(256) void k_bwd_reverse(const BwdArgs a) {
  typedef Walk<DK, DV, T> W;
  typedef typename W::F F;
  __shared__ __attribute__((aligned(16))) T sK[BC * W::LD], sQ[BC * W::LD];
  __shared__ __attribute__((aligned(16))) float part[W::NQ * 4 * 256];
  __shared__ __attribute__((aligned(16))) T sY[2 * W::NT * 512], sX[2 * W::NT * 512],
      sO[2 * W::NT * 512];
  int n0;
  const int64_t sh = W::head_of(n0);
  if (sh >= (int64_t)a.nseq * a.Hv) return;  // the whole workgroup, before any barrier
  const int s = (int)(sh / a.Hv);
  const int h = (int)(sh - (int64_t)s * a.Hv), hk = h / (a.Hv / a.Hk);
  const Seq sq(a, s);
  const int wv = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), nc = sq.chunks();
  const Lane ln = lane_here();
  const int l = ln.id, g = ln.g(), c = ln.c(), r0 = 16 * wv + 4 * g;
  const bool owner = wv < W::NQ;
  const int64_t kld = (int64_t)a.Hk * DK, vld = (int64_t)a.Hv * DV;
  uint32_t koff[W::KI], voff[4];  // byte offsets of this thread's rows of K and Q, of dO
#pragma unroll
  for (int i = 0; i < W::KI; ++i)
    koff[i] = (threadIdx.x + 256 * i) / W::CPR * (uint32_t)kld * sizeof(T);
#pragma unroll
  for (int v = 0; v < 4; ++v) voff[v] = (r0 + v) * (uint32_t)vld * sizeof(T);
  f32x4 st[2];
  W::state_in(st, a.dSf ? a.dSf + sh * DK * DV : nullptr, n0, wv);
  auto tile = [&](int ck) { return a.ws + ((sq.base + ck) * a.Hv + h) * ws_tile(DK, DV); };
  auto rows = [&](int ck) { return min(BC, sq.len - ck * BC); };
  auto vat = [&](int ck) { return ((sq.t0 + (int64_t)ck * BC) * a.Hv + h) * DV + n0; };
  struct Ops {
    RawBlock<T> o;
    f32x4 r, beta, eg, er;
    float el;
    typename W::TRow t;
  };
  auto fetch = [&](Ops& x, int ck) __attribute__((always_inline)) {
    const float* ws = tile(ck);
    const float* rv = ws + ws_rows();
    W::fetch_t(x.t, ws + ws_Tt() + TS * tt_slot(wv, wv / 2), 2 - wv / 2, l);
#pragma unroll
    for (int v = 0; v < 4; ++v) x.r[v] = ws[ws_R() + (uint32_t)(r0 * DV + n0 + c) + v * DV];
    x.o = W::fetch_col((const T*)a.dO + vat(ck), voff, (rows(ck) - 1) * (uint32_t)vld * sizeof(T));
    x.beta = at4(rv + r0);
    x.eg = at4(rv + BC + r0);
    x.er = at4(rv + 2 * BC + r0);
    x.el = rv[2 * BC - 1];
  };
  auto keys = [&](typename W::Rows& x, const void* p, int ck) __attribute__((always_inline)) {
    W::fetch(x, (const T*)p + ((sq.t0 + (int64_t)ck * BC) * a.Hk + hk) * DK, koff,
             (rows(ck) - 1) * (uint32_t)kld * sizeof(T));
  };
  if (nc > 0) {
    Ops ops[2];
    typename W::Rows krs[2], qrs[2];
    keys(krs[0], a.K, nc - 1);
    fetch(ops[0], nc - 1);
    keys(qrs[0], a.Q, nc - 1);
    W::put(sK, krs[0], rows(nc - 1));
    keys(krs[0], a.K, max(nc - 2, 0));
    fetch(ops[1], max(nc - 2, 0));
    keys(qrs[1], a.Q, max(nc - 2, 0));
    keys(krs[1], a.K, max(nc - 3, 0));
    lds_only_barrier();
    auto step = [&](int ck, Ops& op, typename W::Rows& kr, typename W::Rows& qr)
        __attribute__((always_inline)) {
      float* ws = tile(ck);
      W::put(sQ, qr, rows(ck));
      keys(qr, a.Q, max(ck - 2, 0));
      __builtin_amdgcn_sched_barrier(0);
      store_half<F>(sO, wv >> 1, wv & 1,
                    split_half<F>(block_of(op.o, 16 * wv, rows(ck)) * op.eg * a.scale), l);
      if (owner) {
        W::state_out(ws + ws_dS(DK, DV), st, n0, wv);
        W::share(sK, split<F>(st[0], st[1]), part, wv, ln);
      }
      lds_only_barrier();
      typename W::Cols kc;
      if (owner) W::cols(kc, sK, wv, ln);
      store_half<F>(sY, wv >> 1, wv & 1,
                    split_half<F>(op.r + op.er * W::sum(part, wv, l)), l);
      lds_only_barrier();
      W::put(sK, kr, rows(max(ck - 1, 0)));
      keys(kr, a.K, max(ck - 3, 0));
      __builtin_amdgcn_sched_barrier(0);
      f32x4 x[2] = {zero4(), zero4()};
      {
        f32x4 z = zero4(), zl = zero4();
#pragma unroll
        for (int p = 0; p < 2; ++p)
          if (p < 2 - wv / 2)
            mma_both<false>(op.t.v[p], load_terms<F>(sY, p + wv / 2, l), z, zl);
        z += zl;
        const f32x4 dx = op.beta * z;
        store_half<F>(sX, wv >> 1, wv & 1, split_half<F>(-op.eg * dx), l);
        const int m = rows(ck);
        W::rows_out(ws + ws_R(), z, n0, r0);
        char* dV = (char*)((T*)a.dV + vat(ck));
#pragma unroll
        for (int v = 0; v < 4; ++v)
          if (r0 + v < m) *(T*)(dV + (voff[v] + (uint32_t)(c * sizeof(T)))) = (T)dx[v];
        if (owner) {
          typename W::Cols qc;
          W::cols(qc, sQ, wv, ln);
#pragma unroll
          for (int p = 0; p < 2; ++p) {
            const Terms<F> o = load_terms<F>(sO, p, l);
#pragma unroll
            for (int hf = 0; hf < 2; ++hf) x[hf] = mma_in<false>(qc.v[hf][p], o, x[hf]);
          }
        }
      }
      const float el = op.el;
      // (chunk 0 again where there is none: its R has become dZ, which no step uses)
      fetch(op, max(ck - 2, 0));
      lds_only_barrier();
      if (owner) {
#pragma unroll
        for (int p = 0; p < 2; ++p) {
          const Terms<F> y = load_terms<F>(sX, p, l);
#pragma unroll
          for (int hf = 0; hf < 2; ++hf) x[hf] = mma_in<false>(kc.v[hf][p], y, x[hf]);
        }
#pragma unroll
        for (int hf = 0; hf < 2; ++hf) st[hf] = st[hf] * el + x[hf];
      }
    };
    for (int ck = nc - 1; ck >= 0; ck -= 2) {
      step(ck, ops[0], krs[0], qrs[0]);
      if (ck > 0) step(ck - 1, ops[1], krs[1], qrs[1]);
    }
  }
  if (a.dS0 && owner) W::state_out(a.dS0 + sh * DK * DV, st, n0, wv);
}

// ---- every chunk: dQ, dK, dbeta, dg; the value heads of a key head in turn
template <int DK, int DV, typename T>
__global__ __launch_bounds__(256) void k_bwd_grads(const BwdArgs a) {
  typedef typename FragOf<T>::type F;
  constexpr int PV = DV + 4, LD = BC + 4, NB = DK / 64;
  // sPE: Z, then dP and E
  __shared__ float sO[BC * PV], sZ[BC * PV], sY[BC * PV], sPE[2 * BC * LD], sr[5][BC];
  __shared__ float sdb[BC], red[2][4][BC], sdg[BC], send[4];
  static_assert(2 * LD >= PV, "");
  float *sP = sPE, *sE = sPE + BC * LD;
  const int64_t slot = blockIdx.x / a.Hk;
  const int hk = (int)(blockIdx.x - slot * a.Hk), gr = a.Hv / a.Hk;
  int64_t t0 = 0;
  const int m = chunk_at(a, slot, t0);
  if (m == 0) return;
  const int wv = threadIdx.x >> 6, g = lane_g(), c = lane_c();
  const int64_t kld = (int64_t)a.Hk * DK, kat = (t0 * a.Hk + hk) * DK;
  // this wave's NB column blocks of K and Q
  f32x4 kf[NB][4], qf[NB][4], sumq[NB][4], sumk[NB][4];
#pragma unroll
  for (int b = 0; b < NB; ++b)
#pragma unroll
    for (int I = 0; I < 4; ++I) {
      const int64_t at = kat + 16 * (NB * wv + b);
      kf[b][I] = col_block((const T*)a.K + at, kld, 16 * I, m);
      qf[b][I] = col_block((const T*)a.Q + at, kld, 16 * I, m);
      sumq[b][I] = sumk[b][I] = zero4();
    }
  for (int h = hk * gr; h < (hk + 1) * gr; ++h) {
    const float* ws = a.ws + (slot * a.Hv + h) * ws_tile(DK, DV);
    const float* S = ws + ws_S(DV);
    const float* dS = ws + ws_dS(DK, DV);
    for (int i = threadIdx.x; i < 5 * BC; i += 256) (&sr[0][0])[i] = ws[ws_rows() + i];
    rows_to_lds<DV, PV>(sO, (const T*)a.dO + (t0 * a.Hv + h) * DV, (int64_t)a.Hv * DV, m);
    __syncthreads();
    {  // 4 threads a row: Z, dZ, and dZ . X
      const int r = threadIdx.x >> 2;
      const float b = sr[0][r];
      float dot = 0.f;
      for (int e = 4 * (threadIdx.x & 3); e < DV; e += 16) {
        const f32x4 x = at4(ws + ws_X(DV) + r * DV + e), z = at4(ws + ws_R() + r * DV + e);
#pragma unroll
        for (int v = 0; v < 4; ++v) dot = __builtin_fmaf(x[v], z[v], dot);
        *(f32x4*)(sPE + r * PV + e) = b * x;
        *(f32x4*)(sZ + r * PV + e) = z;
      }
      dot += __shfl_xor(dot, 1);
      dot += __shfl_xor(dot, 2);
      if ((threadIdx.x & 3) == 0) sdb[r] = dot;
    }
    __syncthreads();
    for (int J = wv; J < DV / 16; J += 4) {  // Y
      f32x4 z[4];
#pragma unroll
      for (int k = 0; k < 4; ++k) z[k] = down4(sPE + (16 * k + 4 * g) * PV + 16 * J + c, PV);
#pragma unroll
      for (int I = 0; I < 4; ++I) {
        f32x4 y = zero4();
#pragma unroll
        for (int k = 0; k <= I; ++k)
          y = mma16(half_of(load_terms<F>((const T*)(ws + ws_T() + TS * t_slot(I, k / 2)), 0, lane_id()), k & 1), z[k], y);
#pragma unroll
        for (int v = 0; v < 4; ++v) sY[(16 * I + 4 * g + v) * PV + 16 * J + c] = y[v];
      }
    }
    __syncthreads();
    for (int b = wv; b < 20; b += 4) {  // dP and E, lower blocks
      const int bb = b >> 1, I = bb < 1 ? 0 : bb < 3 ? 1 : bb < 6 ? 2 : 3, J = bb - I * (I + 1) / 2;
      const float* left = b & 1 ? sZ : sO;
      f32x4 x = zero4();
#pragma unroll
      for (int k = 0; k < DV / 16; ++k)
        x = mma16(at4(left + (16 * I + c) * PV + 16 * k + 4 * g),
                  at4(sY + (16 * J + c) * PV + 16 * k + 4 * g), x);
#pragma unroll
      for (int v = 0; v < 4; ++v) {
        const int i = 16 * I + 4 * g + v, j = 16 * J + c;
        const float d = i >= j ? expf((sr[3][i] - sr[3][j]) + (sr[4][i] - sr[4][j])) : 0.f;
        if (b & 1)
          sE[i * LD + j] = i > j ? -x[v] * d : 0.f;
        else
          sP[i * LD + j] = i >= j ? a.scale * x[v] * d : 0.f;
      }
    }
    __syncthreads();
    f32x4 dotF[4], dotG[4];
    float end = 0.f, ss = 0.f;
#pragma unroll
    for (int I = 0; I < 4; ++I) dotF[I] = dotG[I] = zero4();
#pragma unroll
    for (int b = 0; b < NB; ++b) {
      const int col = 16 * (NB * wv + b);
      f32x4 dq[4], zs[4], yd[4];
#pragma unroll
      for (int I = 0; I < 4; ++I) dq[I] = zs[I] = yd[I] = zero4();
#pragma unroll 2
      for (int k = 0; k < DV / 16; ++k) {  // dO S^T, dZ S^T, Y dS^T
        const f32x4 sv = at4(S + (int64_t)(col + c) * DV + 16 * k + 4 * g);
        const f32x4 dv = at4(dS + (int64_t)(col + c) * DV + 16 * k + 4 * g);
#pragma unroll
        for (int v = 0; v < 4; ++v) ss = __builtin_fmaf(sv[v], dv[v], ss);
#pragma unroll
        for (int I = 0; I < 4; ++I) {
          const int at = (16 * I + c) * PV + 16 * k + 4 * g;
          dq[I] = mma16(at4(sO + at), sv, dq[I]);
          zs[I] = mma16(at4(sZ + at), sv, zs[I]);
          yd[I] = mma16(at4(sY + at), dv, yd[I]);
        }
      }
#pragma unroll
      for (int I = 0; I < 4; ++I) {
        const int r0 = 16 * I + 4 * g;
        const f32x4 bt = at4(&sr[0][r0]), eg = at4(&sr[1][r0]);
        dq[I] = dq[I] * eg * a.scale;
        f32x4 F = zero4(), R = at4(&sr[2][r0]) * yd[I], km;
#pragma unroll
        for (int k = 0; k <= I; ++k) {
          const int at = (16 * I + c) * LD + 16 * k + 4 * g;
          dq[I] = mma16(at4(sP + at), kf[b][k], dq[I]);
          F = mma16(at4(sE + at), kf[b][k], F);
        }
        km = R;
#pragma unroll
        for (int k = I; k < 4; ++k) {
          const int at = (16 * k + 4 * g) * LD + 16 * I + c;
          km = mma16(down4(sP + at, LD), qf[b][k], km);
          km = mma16(down4(sE + at, LD), at4(&sr[0][16 * k + 4 * g]) * kf[b][k], km);
        }
        const f32x4 kp = bt * (F - eg * zs[I]);
        dotF[I] += kf[b][I] * F;
        dotG[I] += qf[b][I] * dq[I] + kf[b][I] * (kp - km);
        sumq[b][I] += dq[I];
        sumk[b][I] += kp + km;
#pragma unroll
        for (int v = 0; v < 4; ++v) end = __builtin_fmaf(kf[b][I][v], R[v], end);
      }
    }
    end = __builtin_fmaf(sr[1][BC - 1], ss, end);
#pragma unroll
    for (int o = 1; o < 64; o <<= 1) end += __shfl_xor(end, o);
#pragma unroll
    for (int I = 0; I < 4; ++I)
#pragma unroll
      for (int v = 0; v < 4; ++v) {
#pragma unroll
        for (int o = 1; o < 16; o <<= 1) {
          dotF[I][v] += __shfl_xor(dotF[I][v], o);
          dotG[I][v] += __shfl_xor(dotG[I][v], o);
        }
        if (c == 0) {
          red[0][wv][16 * I + 4 * g + v] = dotF[I][v];
          red[1][wv][16 * I + 4 * g + v] = dotG[I][v];
        }
      }
    if (lane_id() == 0) send[wv] = end;
    __syncthreads();
    if (threadIdx.x < BC) {
      const int r = threadIdx.x;
      float dg = (red[1][0][r] + red[1][1][r]) + (red[1][2][r] + red[1][3][r]);
      if (r == m - 1) dg += (send[0] + send[1]) + (send[2] + send[3]);
      sdg[r] = dg;
      if (r < m)
        a.dbeta[(t0 + r) * a.Hv + h] =
            sdb[r] + ((red[0][0][r] + red[0][1][r]) + (red[0][2][r] + red[0][3][r]));
    }
    __syncthreads();
    if (threadIdx.x < m) {
      const int r = threadIdx.x;
      float dg = sdg[r];
      // the last g of a part of C tokens is in the gamma of every later row
      if (a.C < BC && r % a.C == a.C - 1)
        for (int i = r + 1; i < m; ++i) dg += sdg[i];
      a.dg[(t0 + r) * a.Hv + h] = dg;
    }
  }
#pragma unroll
  for (int b = 0; b < NB; ++b)
#pragma unroll
    for (int I = 0; I < 4; ++I)
#pragma unroll
      for (int v = 0; v < 4; ++v) {
        const int r = 16 * I + 4 * g + v;
        if (r < m) {
          const int64_t at = kat + r * kld + 16 * (NB * wv + b) + c;
          ((T*)a.dQ)[at] = (T)sumq[b][I][v];
          ((T*)a.dK)[at] = (T)sumk[b][I][v];
        }
      }
}

int64_t backward_slots(int nseq, int L, bool packed) {
  return packed ? (int64_t)L / BC + nseq : (int64_t)nseq * ((L + BC - 1) / BC);
}
int64_t backward_tile_bytes(int dk, int dv) { return ws_tile(dk, dv) * 4; }

template <int DK, int DV, typename T>
static hipError_t run_backward(const BwdArgs& a, int64_t slots, hipStream_t st) {
  const unsigned walks = (unsigned)(((int64_t)a.nseq * a.Hv + 7) / 8 * 8 * (DV / 16));
  if (slots > 0) {
    hipLaunchKernelGGL((k_bwd_prep<DK, DV, T>), dim3((unsigned)(slots * a.Hv)), dim3(256), 0, st, a);
    hipLaunchKernelGGL((k_bwd_states<DK, DV, T>), dim3(walks), dim3(256), 0, st, a);
  }
  if (slots > 0 || a.dS0)
    hipLaunchKernelGGL((k_bwd_reverse<DK, DV, T>), dim3(walks), dim3(256), 0, st, a);
  if (slots > 0)
    hipLaunchKernelGGL((k_bwd_grads<DK, DV, T>), dim3((unsigned)(slots * a.Hk)), dim3(256), 0, st, a);
  return hipGetLastError();
}

hipError_t launch_backward(const void* Q, const void* K, const void* V, const float* beta,
                           const float* g, const void* dO, const float* S0, const float* dSf,
                           void* dQ, void* dK, void* dV, float* dbeta, float* dg, float* dS0,
                           float* ws, const int* cu, int nseq, int L, int Hk, int Hv, int dk,
                           int dv, int C, float scale, int dtype, hipStream_t st) {
  BwdArgs a{Q,  K,     V,  dO,  beta, g,  S0,   dSf, dQ,              dK, dV, dbeta,
            dg, dS0,   ws, cu,  nseq, L,  (L + BC - 1) / BC, Hk, Hv, C, scale};
  const int64_t slots = L > 0 ? backward_slots(nseq, L, cu != nullptr) : 0;
  GDN_DK_SWITCH(dk, GDN_DV_SWITCH(dv, {
    return dtype == 0 ? run_backward<DK, DV, float>(a, slots, st)
                      : run_backward<DK, DV, __bf16>(a, slots, st);
  }))
  return hipErrorNotSupported;
}

}  // namespace gdn
