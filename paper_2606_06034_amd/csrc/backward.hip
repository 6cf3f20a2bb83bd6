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
#include "forward.hpp"
#include "launch.hpp"
#include "layer.hpp"
#include "split.hpp"

namespace gdn {

namespace {

constexpr int BC = 64;  // tokens a chunk

// Workspace of one (chunk, value head), in floats.  T and T^T lie as the terms
// (split.hpp) of the pair fragments of their row blocks, 3 KB a fragment (2 KB
// with fp32 inputs): T (I, p) with 2p <= I, T^T (I, p) with 2p + 1 >= I.
// X, R and dZ lie as column-form blocks, S and dS as row-form blocks (tile16.hpp),
// the 4 values of a lane side by side: 1 KB a block, read and written whole.
constexpr int TS = 768;
__host__ __device__ constexpr int blk_at(int I, int J, int NJ) { return (I * NJ + J) * 256; }
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
        *(f32x4*)(ws + ws_R() + blk_at(I, J, DV / 16) + 4 * lane_id()) = x;
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
  // the same as row-form blocks, transposed through this wave's part of LDS
  static constexpr int TB = 16 * 20;
  static __device__ __forceinline__ void blocks_out(float* p, const f32x4 (&st)[2], int n0, int wv,
                                                    float* t, Lane ln) {
#pragma unroll
    for (int h = 0; h < 2; ++h)
#pragma unroll
      for (int v = 0; v < 4; ++v) t[TB * h + (4 * ln.g() + v) * 20 + ln.c()] = st[h][v];
    lds_sync<true>();
#pragma unroll
    for (int h = 0; h < 2; ++h)
      *(f32x4*)(p + blk_at(2 * wv + h, n0 / 16, NS) + 4 * ln.id) =
          at4(t + TB * h + ln.c() * 20 + 4 * ln.g());
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
  __shared__ __attribute__((aligned(16))) float sT[W::NQ][2 * W::TB];
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
      W::blocks_out(ws + ws_S(DV), st, n0, wv, sT[wv], ln);
      W::share(sK, split<F>(st[0], st[1]), part, wv, ln);
    }
    lds_only_barrier();
    typename W::Cols kc;
    if (owner) W::cols(kc, sK, wv, ln);
    {
      const f32x4 x = block_of(op.v, 16 * wv, rows(ck)) - op.eg * W::sum(part, wv, l);
      *(f32x4*)(ws + ws_X(DV) + blk_at(wv, n0 / 16, W::NS) + 4 * l) = x;
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
  __shared__ __attribute__((aligned(16))) float sT[W::NQ][2 * W::TB];
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
    x.r = at4(ws + ws_R() + blk_at(wv, n0 / 16, W::NS) + 4 * l);
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
        W::blocks_out(ws + ws_dS(DK, DV), st, n0, wv, sT[wv], ln);
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
        *(f32x4*)(ws + ws_R() + blk_at(wv, n0 / 16, W::NS) + 4 * l) = z;
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
// Eight waves.  Wave w has the 32 feature columns 32 (w % (DK / 32)) of dQ and dK
// for NR row blocks of the chunk.  dO, dZ and Y lie in LDS as pair fragments along
// the value columns (one form serves as left operand and, transposed, as right
// one); S and dS come from memory as right operands, each value split into
// terms by the waves that use it.  The blocks of dP and E wait in registers until the
// products with the states are done, and then take the place of dO and dZ.
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

// sum over the 16 lanes of a row of the wave
__device__ __forceinline__ float sum16(float x) {
  auto add = [&](int y) { x += __builtin_bit_cast(float, y); };
  add(__builtin_amdgcn_mov_dpp(__builtin_bit_cast(int, x), 0xB1, 0xf, 0xf, true));   // lane ^ 1
  add(__builtin_amdgcn_mov_dpp(__builtin_bit_cast(int, x), 0x4E, 0xf, 0xf, true));   // lane ^ 2
  add(__builtin_amdgcn_mov_dpp(__builtin_bit_cast(int, x), 0x141, 0xf, 0xf, true));  // 7 - lane
  add(__builtin_amdgcn_mov_dpp(__builtin_bit_cast(int, x), 0x140, 0xf, 0xf, true));  // 15 - lane
  return x;
}

template <int DK, int DV, typename T>
__global__ __launch_bounds__(512) void k_bwd_grads(const BwdArgs a) {
  typedef Grads<DK, DV, T> G;
  typedef typename G::F F;
  constexpr int NT = G::NT, NP = G::NP, NR = G::NR, LDK = G::LDK;
  constexpr int E = 16 / sizeof(T), NJ = DV / 16, RY = 8 / NJ;
  typedef T Vec __attribute__((ext_vector_type(E)));
  __shared__ __attribute__((aligned(16))) T sm[G::SIZE];
  __shared__ __attribute__((aligned(16))) float sr[5][BC];
  __shared__ __attribute__((aligned(16))) float tr[8][16 * 20];
  __shared__ float sdb[NJ][BC], red[2][G::NC][BC], sdg[BC], send[8];
  const int64_t slot = blockIdx.x / a.Hk;
  const int hk = (int)(blockIdx.x - slot * a.Hk), gr = a.Hv / a.Hk;
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
    float* ws = a.ws + (slot * a.Hv + h) * ws_tile(DK, DV);
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
      float* t = tr[wv];
#pragma unroll
      for (int I = 0; I < 4; ++I) {
        if (I % RY != wv / NJ) continue;
#pragma unroll
        for (int v = 0; v < 4; ++v) {
          t[(4 * g + v) * 20 + c] = zb[I][v];
          const float d = sum16(xb[I][v] * zb[I][v]);
          if (c == 0) sdb[J][16 * I + 4 * g + v] = d;
        }
        lds_sync<true>();
        store_half<F>(sm + G::oZ, I * NP + (J >> 1), J & 1, split_half<F>(at4(t + c * 20 + 4 * g)), l);
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
    // ---- Y = T Z: value column block J of the rows I % RY
#pragma unroll
    for (int I = 0; I < 4; ++I) {
      if (I % RY != wv / NJ) continue;
      f32x4 y = zero4(), yl = zero4();
#pragma unroll
      for (int p = 0; p <= I / 2; ++p)
        mma_both<true>(load_terms<F>(sm + G::oT, t_slot(I, p), l), z[p], y, yl);
      store_half<F>(sm + G::oY, I * NP + (J >> 1), J & 1, split_half<F>(y + yl), l);
    }
    States st;
    states(st, 0);
    __syncthreads();
    // ---- dP and E, a lower block each; an E block costs as much as two of dP
    struct Blk {
      int kind, I, J;  // kind: 0 dP, 1 E, -1 none
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
      const int I = n < 1 ? 0 : n < 3 ? 1 : n < 6 ? 2 : 3;
      return Blk{kind, I, n - I * (I + 1) / 2};
    };
    f32x4 pe[3];
#pragma unroll
    for (int i = 0; i < 3; ++i) {
      __builtin_amdgcn_sched_barrier(0);
      const Blk k = block(i);
      f32x4 x = zero4(), xl = zero4();
      if (k.kind == 1) {
#pragma unroll 1
        for (int p = 0; p < NP; ++p)
          mma_both<false>(load_terms<F>(sm + G::oZ, k.I * NP + p, l),
                          load_terms<F>(sm + G::oY, k.J * NP + p, l), x, xl);
      } else if (k.kind == 0) {
#pragma unroll 1
        for (int p = 0; p < NP; ++p)
          x = mma_in<false>(slot_load<F>(sm + G::oO + (k.I * NP + p) * 512, l),
                            load_terms<F>(sm + G::oY, k.J * NP + p, l), x);
      }
      x += xl;
#pragma unroll
      for (int v = 0; v < 4; ++v) {
        const int r = 16 * k.I + 4 * g + v, j = 16 * k.J + c;
        const float d = r >= j ? expf((sr[3][r] - sr[3][j]) + (sr[4][r] - sr[4][j])) : 0.f;
        pe[i][v] = k.kind == 1 ? (r > j ? -x[v] * d : 0.f) : a.scale * x[v] * d;
      }
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
        for (int b = 0; b < 2; ++b) {
          dq[b][i] = mma_in<false>(o, sv[b], dq[b][i]);
          zs[b][i] = mma_both<false>(z, sv[b], zs[b][i]);
          yd[b][i] = mma_both<false>(y, dv[b], yd[b][i]);
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
      const Blk k = block(i);
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
    float* acc = a.ws + (slot * a.Hv + hk * gr) * ws_tile(DK, DV) + ws_S(DV) + 4 * tid;
    float end = 0.f;
#pragma unroll
    for (int i = 0; i < NR; ++i) {
      const int I = I0 + i, r0 = 16 * I + 4 * g;
      const f32x4 bt = at4(&sr[0][r0]), eg = at4(&sr[1][r0]), er = at4(&sr[2][r0]);
      f32x4 F_[2], km[2], R[2];
#pragma unroll
      for (int b = 0; b < 2; ++b) {
        dq[b][i] = dq[b][i] * eg * a.scale;
        F_[b] = zero4();
        R[b] = km[b] = er * yd[b][i];
      }
#pragma unroll
      for (int p = 0; p < 2; ++p) {
        if (p <= I / 2) {
          const Terms<F> P = load_terms<F>(sm + G::oPr, t_slot(I, p), l);
          const Terms<F> Er = load_terms<F>(sm + G::oEr, t_slot(I, p), l);
#pragma unroll
          for (int b = 0; b < 2; ++b) {
            dq[b][i] = mma_in<false>(P, kf[b][p], dq[b][i]);
            F_[b] = mma_in<false>(Er, kf[b][p], F_[b]);
          }
        }
        if (p >= I / 2) {
          const Terms<F> P = load_terms<F>(sm + G::oPc, tt_slot(I, p), l);
          const Terms<F> Ec = load_terms<F>(sm + G::oEc, tt_slot(I, p), l);
#pragma unroll
          for (int b = 0; b < 2; ++b) {
            km[b] = mma_in<false>(P, qf[b][p], km[b]);
            km[b] = mma_in<false>(Ec, kf[b][p], km[b]);
          }
        }
      }
      f32x4 dotF = zero4(), dotG = zero4();
#pragma unroll
      for (int b = 0; b < 2; ++b) {
        const f32x4 kp = bt * (F_[b] - eg * zs[b][i]);
        // the rows' own k and q, from the pair that holds their block
        const Pair<F> kk = I < 2 ? kf[b][0] : kf[b][1], qq = I < 2 ? qf[b][0] : qf[b][1];
        const f32x4 k = I & 1 ? kk.hi() : kk.lo(), q = I & 1 ? qq.hi() : qq.lo();
        dotF += k * F_[b];
        dotG += q * dq[b][i] + k * (kp - km[b]);
#pragma unroll
        for (int v = 0; v < 4; ++v) end = __builtin_fmaf(k[v], R[b][v], end);
        f32x4 sq = dq[b][i], sk = kp + km[b];
        float* at = acc + (b * NR + i) * 2 * 2048;
        if (h > hk * gr) {
          sq += at4(at);
          sk += at4(at + 2048);
        }
        if (h + 1 < (hk + 1) * gr) {
          *(f32x4*)at = sq;
          *(f32x4*)(at + 2048) = sk;
        } else {
#pragma unroll
          for (int v = 0; v < 4; ++v)
            if (r0 + v < m) {
              const int64_t to = kat + (r0 + v) * kld + col + 16 * b + c;
              ((T*)a.dQ)[to] = (T)sq[v];
              ((T*)a.dK)[to] = (T)sk[v];
            }
        }
      }
#pragma unroll
      for (int v = 0; v < 4; ++v) {
        const float f = sum16(dotF[v]), d = sum16(dotG[v]);
        if (c == 0) {
          red[0][wv % G::NC][r0 + v] = f;
          red[1][wv % G::NC][r0 + v] = d;
        }
      }
    }
    // (every row group has formed the same <S, dS> of its columns)
    if (I0 == 0) end = __builtin_fmaf(sr[1][BC - 1], ss, end);
    end = sum16(end);
    end += __shfl_xor(end, 16);
    end += __shfl_xor(end, 32);
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
    if (tid < m) {
      const int r = tid;
      float dg = sdg[r];
      // the last g of a part of C tokens is in the gamma of every later row
      if (a.C < BC && r % a.C == a.C - 1)
        for (int i = r + 1; i < m; ++i) dg += sdg[i];
      a.dg[(t0 + r) * a.Hv + h] = dg;
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
    hipLaunchKernelGGL((k_bwd_grads<DK, DV, T>), dim3((unsigned)(slots * a.Hk)), dim3(512), 0, st, a);
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
