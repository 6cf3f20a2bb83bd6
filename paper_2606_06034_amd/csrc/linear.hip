// linear.hip -- linear attention with a decay for each head, chunked, and its gradients.
//
// With a_t = e^{g_t}, S_t = a_t S_{t-1} + k_t v_t^T, o_t = scale S_t^T q_t.  In a chunk of 64
// tokens, H the cumulative g up to and with a token, D_ij = e^{H_i - H_j} (j <= i),
//   O = s_out diag(e^H) Q S + scale ((Q K^T) (.) D) V,
//   S' = e^total S + (s_in diag(e^{total - H}) K)^T V          (s_out = scale, s_in = 1).
// The gradients are three passes of the same form over other operands:
//   dQ: Q <- dO, K <- V, V <- K, states S^T;
//   dK: Q <- V, K <- dO, V <- Q and dV: Q <- K, K <- Q, V <- dO in reversed time, states dS^T
//   and dS (the gradient of the state leaving the chunk), s_out = 1, s_in = scale.
// Reversed, row r is the chunk's token m - 1 - r, and with H the sum of g over the rows
// before r all of the above holds as it stands.  The gradient of g is
//   dg_t = sum over i >= t of (q_i . dQ_i - k_i . dK_i) + <S, dS> at the end of the segment.
// What tokens of one chunk give each other cancels in that sum past the chunk, so that only
// what came through the states is carried from chunk to chunk (else the roundings of a whole
// segment pile up on the gradients of fast-forgetting heads).
//
// A sequence is cut into segments, which workgroups walk chunk by chunk with the state in
// registers.  More than one segment: k_lin_state forms what each adds to the state,
// k_lin_scan carries the states over the segments, k_lin_forward / k_lin_backward walk.
//
// Precision.  bf16 inputs are exact operands of the matrix instructions; fp32 factors
// (states, decayed values, P) enter as sums of bf16 terms (split.hpp).
#include <algorithm>

#include "lanes.hpp"
#include "launch.hpp"
#include "layer.hpp"
#include "linear.hpp"
#include "split.hpp"

namespace gdn {

namespace {

template <typename T> struct FragFor { typedef f32x4 type; };
template <> struct FragFor<__bf16> { typedef bf16x4 type; };

constexpr double kLog2e = 1.4426950408889634074;

template <int CTRL, int ROWS>
__device__ __forceinline__ double moved_or_zero(double x) {
  const uint64_t u = __builtin_bit_cast(uint64_t, x);
  const uint32_t lo = __builtin_amdgcn_update_dpp(0, (int)(uint32_t)u, CTRL, ROWS, 0xf, false);
  const uint32_t hi = __builtin_amdgcn_update_dpp(0, (int)(uint32_t)(u >> 32), CTRL, ROWS, 0xf,
                                                  false);
  return __builtin_bit_cast(double, (uint64_t)hi << 32 | lo);
}
// sums over a lane and those before it
__device__ __forceinline__ double prefix64(double x) {
  x += moved_or_zero<0x111, 0xf>(x);  // the lane 1, 2, 4, 8 before, of 16
  x += moved_or_zero<0x112, 0xf>(x);
  x += moved_or_zero<0x114, 0xf>(x);
  x += moved_or_zero<0x118, 0xf>(x);
  x += moved_or_zero<0x142, 0xa>(x);  // lane 15 of the 16 before, into the second and fourth
  x += moved_or_zero<0x143, 0xc>(x);  // lane 31, into the upper half
  return x;
}
__device__ __forceinline__ double lane63(double x) {
  const uint64_t u = __builtin_bit_cast(uint64_t, x);
  const uint32_t lo = __builtin_amdgcn_readlane((uint32_t)u, 63);
  const uint32_t hi = __builtin_amdgcn_readlane((uint32_t)(u >> 32), 63);
  return __builtin_bit_cast(double, (uint64_t)hi << 32 | lo);
}
// 2^x, x in two parts as it is rounded
__device__ __forceinline__ float exp2_of(double x) {
  const float hi = (float)x, lo = (float)(x - (double)hi), e = __builtin_amdgcn_exp2f(hi);
  return __builtin_fmaf(e, lo * 0.69314718f, e);
}

// The decays of a chunk's rows, in LDS.  The sums run in 64 bits, and H is kept as two floats:
// differences of rows of a fast-forgetting head are small beside the sums themselves.
// A log-decay of -inf (forget all) counts as -1e4, whose exponential is 0 as well and whose
// differences are numbers.
struct Gates {
  float hi[LC], lo[LC], out[LC], in[LC];  // H in units of log 2; s_out e^H, s_in e^{total - H}
  float el, pad[3];                       // e^total
};
__device__ __forceinline__ double log_decay(float g) {
  return (double)(g < -1e4f ? -1e4f : g) * kLog2e;
}
// wave-wide: row l of m, `g` its token's (per_token) or the head's; returns the total
__device__ __forceinline__ double form_gates(Gates* s, float g, bool per_token, int m, bool rev,
                                             float s_out, float s_in) {
  const int l = lane_id();
  double H, total;
  if (per_token) {
    const double d = l < m ? log_decay(g) : 0.0;
    H = prefix64(d);
    total = lane63(H);
    if (rev) H -= d;
  } else {
    const double d = log_decay(g);
    H = d * min(rev ? l : l + 1, m);
    total = d * m;
  }
  const float hi = (float)H;
  s->hi[l] = hi;
  s->lo[l] = (float)(H - (double)hi);
  s->out[l] = s_out * exp2_of(H);
  s->in[l] = s_in * exp2_of(total - H);
  if (l == 0) s->el = exp2_of(total);
  return total;
}

// A chunk's rows of one head on the way from memory to LDS: 16-byte pieces, 256 threads.
template <int D, typename T>
struct Rows {
  static constexpr int E = 16 / sizeof(T), CPR = D / E, N = LC * CPR / 256, LD = D + E;
  typedef T Vec __attribute__((ext_vector_type(E)));
  Vec v[N];
  // p: the chunk's first token, ld values a token; rows past m repeat one of its own
  __device__ __forceinline__ void load(const T* __restrict__ p, uint32_t ld, int m, bool rev) {
#pragma unroll
    for (int i = 0; i < N; ++i) {
      const int at = threadIdx.x + 256 * i, r = min(at / CPR, m - 1);
      v[i] = *(const Vec*)(p + ((uint32_t)(rev ? m - 1 - r : r) * ld + at % CPR * E));
    }
  }
  __device__ __forceinline__ void store(T* s, int m) const {
#pragma unroll
    for (int i = 0; i < N; ++i) {
      const int at = threadIdx.x + 256 * i, r = at / CPR;
      *(Vec*)(s + r * LD + at % CPR * E) = r < m ? v[i] : Vec{};
    }
  }
};

// Fragments from LDS rows, LD values apart.  Along a row: slot s of lane (g, c) is value
// 8g + s of the run at c0 of row r0 + c.  Down the rows: slot s is row r0 + 16 (s / 4) + 4g +
// s % 4 of column c0 + GS (c / 4) + c % 4.
template <int LD>
__device__ __forceinline__ Pair<bf16x4> run_frag(const __bf16* s, int r0, int c0, Lane ln) {
  return Pair<bf16x4>{*(const bf16x8*)(s + (r0 + ln.c()) * LD + c0 + 8 * ln.g())};
}
template <int LD>
__device__ __forceinline__ Pair<f32x4> run_frag(const float* s, int r0, int c0, Lane ln) {
  const float* p = s + (r0 + ln.c()) * LD + c0 + 8 * ln.g();
  return join(*(const f32x4*)p, *(const f32x4*)(p + 4));
}
template <int LD, int GS>
__device__ __forceinline__ Pair<bf16x4> down_frag(const __bf16* s, int r0, int c0, Lane ln) {
  const __bf16* p = s + (r0 + 4 * ln.g() + (ln.c() >> 2)) * LD + c0 + GS * (ln.c() & 3);
  return join(read_transposed(p), read_transposed(p + 16 * LD));
}
template <int LD, int GS>
__device__ __forceinline__ Pair<f32x4> down_frag(const float* s, int r0, int c0, Lane ln) {
  const float* p = s + (r0 + 4 * ln.g()) * LD + c0 + GS * (ln.c() >> 2) + (ln.c() & 3);
  f32x4 a, b;
#pragma unroll
  for (int v = 0; v < 4; ++v) a[v] = p[v * LD], b[v] = p[(16 + v) * LD];
  return join(a, b);
}

// The first N terms of a split value (fp32: the value)
template <typename F, int N> struct Some { Pair<F> t[N]; };
template <typename F, int N> constexpr int kTerms = TermsOf<F>::N == 1 ? 1 : N;
template <typename F, int N>
__device__ __forceinline__ auto some(f32x4 lo, f32x4 hi) {
  constexpr int M = kTerms<F, N>;
  Some<F, M> r;
  if constexpr (TermsOf<F>::N == 1) {
    r.t[0] = join(lo, hi);
  } else {
    typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
    float a = lo[0], b = lo[1], c = lo[2], d = lo[3], e = hi[0], f = hi[1], x = hi[2], y = hi[3];
#pragma unroll
    for (int i = 0; i < M; ++i) {
      const uint32_t p = take2(a, b), q = take2(c, d), u = take2(e, f), w = take2(x, y);
      r.t[i].v = __builtin_bit_cast(bf16x8, u32x4{p, q, u, w});
    }
  }
  return r;
}

// A wave's part of a [DK, DV] state: all rows, NS blocks of 16 columns.  Block m = 2q + h,
// block row 4g + v holds state row 32q + 8g + 4h + v, so that two blocks are the pair that
// meets a run of 8 values of a row; column c of block n is 16 NS w + 4 NS (c / 4) + 4n + c % 4,
// so that a row-form result has 4 NS neighbouring columns a lane.
template <int DK, int DV>
struct StateOf {
  static constexpr int NS = DV / 64, NQ = DK / 32;
  f32x4 b[2 * NQ][NS];
  static __device__ __forceinline__ int row(int m, Lane ln) {
    return 32 * (m >> 1) + 8 * ln.g() + 4 * (m & 1);
  }
  static __device__ __forceinline__ int col(int n, int w, Lane ln) {
    return 16 * NS * w + 4 * NS * (ln.c() >> 2) + 4 * n + (ln.c() & 3);
  }
  __device__ __forceinline__ void zero() {
#pragma unroll
    for (int m = 0; m < 2 * NQ; ++m)
#pragma unroll
      for (int n = 0; n < NS; ++n) b[m][n] = zero4();
  }
  // memory holds rows of DV values, or with `flip` the transposed state, rows of DK
  __device__ __forceinline__ void load(const float* p, bool flip, int w, Lane ln) {
#pragma unroll
    for (int m = 0; m < 2 * NQ; ++m)
#pragma unroll
      for (int n = 0; n < NS; ++n) {
        const int r = row(m, ln), c = col(n, w, ln);
        if (flip) {
          b[m][n] = *(const f32x4*)(p + c * DK + r);
        } else {
#pragma unroll
          for (int v = 0; v < 4; ++v) b[m][n][v] = p[(r + v) * DV + c];
        }
      }
  }
  __device__ __forceinline__ void store(float* p, bool flip, int w, Lane ln) const {
#pragma unroll
    for (int m = 0; m < 2 * NQ; ++m)
#pragma unroll
      for (int n = 0; n < NS; ++n) {
        const int r = row(m, ln), c = col(n, w, ln);
        if (flip) {
          *(f32x4*)(p + c * DK + r) = b[m][n];
        } else {
#pragma unroll
          for (int v = 0; v < 4; ++v) p[(r + v) * DV + c] = b[m][n][v];
        }
      }
  }
  // S <- el S + (diag(in) K)^T V of the chunk in LDS, the factor on V's rows
  template <int TS, typename T>
  __device__ __forceinline__ void update(const T* sK, const T* sV, const Gates* gt, int w,
                                         Lane ln) {
    typedef typename FragFor<T>::type F;
    constexpr int LDK = Rows<DK, T>::LD, LDV = Rows<DV, T>::LD;
    const float el = gt->el;
#pragma unroll
    for (int m = 0; m < 2 * NQ; ++m)
#pragma unroll
      for (int n = 0; n < NS; ++n) b[m][n] *= el;
#pragma unroll
    for (int p = 0; p < 2; ++p) {
      const f32x4 wl = *(const f32x4*)(gt->in + 32 * p + 4 * ln.g());
      const f32x4 wh = *(const f32x4*)(gt->in + 32 * p + 16 + 4 * ln.g());
      Some<F, kTerms<F, TS>> y[NS];
#pragma unroll
      for (int n = 0; n < NS; ++n) {
        const Pair<F> x = down_frag<LDV, 4 * NS>(sV, 32 * p, 16 * NS * w + 4 * n, ln);
        y[n] = some<F, TS>(x.lo() * wl, x.hi() * wh);
      }
#pragma unroll
      for (int m = 0; m < 2 * NQ; ++m) {
        const Pair<F> k = down_frag<LDK, 8>(sK, 32 * p, 32 * (m >> 1) + 4 * (m & 1), ln);
#pragma unroll
        for (int i = kTerms<F, TS> - 1; i >= 0; --i)
#pragma unroll
          for (int n = 0; n < NS; ++n)
            b[m][n] = Pair<F>::template mma<false>(k, y[n].t[i], b[m][n]);
      }
    }
  }
};

// The tokens of a segment
struct Segment {
  int64_t t0;   // its first token
  int len;      // its tokens (0: nothing to do)
  int s, j, n;  // sequence, and which segment of how many
  __device__ Segment(const LinSeqs& q, uint32_t slot) {
    int64_t base;
    int all;
    s = q.find(slot);
    q.at(s, t0, base, all);
    const int64_t at = (int64_t)slot - base, skip = at * q.seg;
    n = q.segments(all);
    len = at < 0 || skip >= all ? 0 : (int)min((int64_t)q.seg, all - skip);
    j = (int)at;
    t0 += skip;
  }
};

// work item of a workgroup: neighbours on one XCD (workgroups go round the 8 in turn)
__device__ __forceinline__ uint32_t work_item(uint32_t b, uint32_t n) {
  return (b & 7) * ((n + 7) >> 3) + (b >> 3);
}

// ---- what a segment adds to the state
template <int DK, int DV, typename T, int TS>
__device__ __forceinline__ void add_of_segment(const LinArgs& a, const Segment& sg, uint32_t slot,
                                               int h, bool rev, T* sK, T* sV, Gates* gt) {
  const int gr = a.Hv / a.Hk;
  const T* K = (const T*)(rev ? a.Q : a.K) + (sg.t0 * a.Hk + h / gr) * DK;
  const T* V = (const T*)(rev ? a.dO : a.V) + (sg.t0 * a.Hv + h) * DV;
  const uint32_t ldk = (uint32_t)a.Hk * DK, ldv = (uint32_t)a.Hv * DV;
  const int w = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const Lane ln = lane_here();
  const int nc = (sg.len + LC - 1) / LC;
  StateOf<DK, DV> S;
  S.zero();
  Rows<DK, T> k;
  Rows<DV, T> v;
  float g = a.per_token ? 0.f : a.g[h];
  auto fetch = [&](int i) __attribute__((always_inline)) {
    const int at = (rev ? nc - 1 - i : i) * LC, m = min(LC, sg.len - at);
    k.load(K + (int64_t)at * ldk, ldk, m, rev);
    v.load(V + (int64_t)at * ldv, ldv, m, rev);
    if (a.per_token && w == 0) {
      const int r = min(ln.id, m - 1);
      g = a.g[(sg.t0 + at + (rev ? m - 1 - r : r)) * a.Hv + h];
    }
  };
  double total = 0.0;
  fetch(0);
  for (int i = 0; i < nc; ++i) {
    const int m = min(LC, sg.len - (rev ? nc - 1 - i : i) * LC);
    lds_only_barrier();
    k.store(sK, m);
    v.store(sV, m);
    if (w == 0) total += form_gates(gt, g, a.per_token, m, rev, 1.f, rev ? a.scale : 1.f);
    if (i + 1 < nc) fetch(i + 1);
    lds_only_barrier();
    S.template update<TS>(sK, sV, gt, w, ln);
  }
  float* to = (rev ? a.R : a.U) + ((int64_t)slot * a.Hv + h) * DK * DV;
  S.store(to, false, w, ln);
  if (threadIdx.x == 0 && (!rev || sg.j == sg.n - 1))  // (once for each segment)
    a.dec[(int64_t)slot * a.Hv + h] = exp2_of(total);
}

}  // namespace

// `both`: the gradients' states too, in the second half of the work items
template <int DK, int DV, typename T, int TS>
__global__ __launch_bounds__(256) void k_lin_state(const LinArgs a, uint32_t n, bool both) {
  __shared__ __attribute__((aligned(16))) T sK[LC * Rows<DK, T>::LD], sV[LC * Rows<DV, T>::LD];
  __shared__ __attribute__((aligned(16))) Gates gt;
  uint32_t w = work_item(blockIdx.x, n * (both ? 2 : 1));
  if (w >= n * (both ? 2 : 1)) return;
  const bool rev = w >= n;
  if (rev) w -= n;
  const uint32_t slot = w / (uint32_t)a.Hv;
  const int h = (int)(w - slot * (uint32_t)a.Hv);
  const Segment sg(a.q, slot);
  // (the last segment's share ends in S_final, the first one's in dS0: the walks form those)
  if (sg.len == 0 || (rev ? sg.j == 0 : sg.j == sg.n - 1)) return;
  add_of_segment<DK, DV, T, TS>(a, sg, slot, h, rev, sK, sV, &gt);
}

// The states carried over the segments of each sequence, in place: U from what a segment
// adds to the state that enters it, R to the gradient of the state that leaves it.
__global__ __launch_bounds__(256) void k_lin_scan(const LinArgs a, int parts) {
  const bool rev = blockIdx.y;
  const int64_t size = (int64_t)a.dk * a.dv, step = a.Hv * size;
  const uint32_t mine = blockIdx.x / (uint32_t)parts;
  const int64_t e = ((int64_t)(blockIdx.x - mine * (uint32_t)parts) * 256 + threadIdx.x) * 4;
  const uint32_t most = (uint32_t)a.q.nseq * (uint32_t)a.Hv;
  for (uint32_t sh = mine; sh < most; sh += gridDim.x / (uint32_t)parts) {
    const uint32_t s = sh / (uint32_t)a.Hv;
    const int h = (int)(sh - s * (uint32_t)a.Hv);
    int64_t t0, base;
    int len;
    a.q.at((int)s, t0, base, len);
    const int n = a.q.segments(len);
    if (n == 0) continue;
    const float* from = rev ? a.dSf : a.S0;
    f32x4 S = from ? *(const f32x4*)(from + (int64_t)sh * size + e) : zero4();
    float* X = (rev ? a.R : a.U) + (base * a.Hv + h) * size + e;
    const float* d = a.dec + base * a.Hv + h;
    constexpr int A = 4;  // asked for ahead
    for (int i0 = 0; i0 < n; i0 += A) {
      f32x4 x[A];
      float f[A];
#pragma unroll
      for (int u = 0; u < A; ++u) {
        const int i = min(i0 + u, n - 2), j = rev ? n - 1 - i : i;
        if (n > 1) {
          x[u] = *(const f32x4*)(X + j * step);
          f[u] = d[(int64_t)j * a.Hv];
        }
      }
#pragma unroll
      for (int u = 0; u < A; ++u) {
        const int i = i0 + u, j = rev ? n - 1 - i : i;
        if (i < n) {
          *(f32x4*)(X + j * step) = S;
          if (i + 1 < n) S = f[u] * S + x[u];
        }
      }
    }
  }
}

namespace {

template <typename T, int N> struct RunType { typedef T type __attribute__((ext_vector_type(N))); };
template <typename T, int N> using RunOf = typename RunType<T, N>::type;

// One pass along a segment for one value head.
struct Pass {
  const void *q, *k, *v, *x;   // x: rows whose products with the result are kept (or null)
  uint32_t ldq, ldk, ldv, ldo; // values a token
  void* out;
  float* acc;                  // sums of a group's heads (null: one head)
  bool first, last;            // of the group
  float* dot;                  // of each row, at the segment's first token
  float* far;                  // of each chunk, of what came from the state
  const float* start;          // the state that enters (or null: zeros)
  float* fin;                  // the state that leaves (or null)
  const float* against;        // [product with the state that leaves] (or null)
  float* anchor;
  bool flip, rev;              // flip: the state's transposed in memory
  float s_out, s_in;
};

template <int DK, int DV, typename T, int TO>
struct PassLds {
  typedef typename FragFor<T>::type F;
  T q[LC * Rows<DK, T>::LD], k[LC * Rows<DK, T>::LD], v[LC * Rows<DV, T>::LD];
  T p[6 * kTerms<F, TO> * 512];
  float dot[4][LC], far[4];
  Gates gt;
};

__host__ __device__ constexpr int p_slot(int I, int p) { return (I == 3 ? 4 : I) + p; }

template <int DK, int DV, typename T, int TS, int TO>
__device__ __forceinline__ void walk(const LinArgs& a, const Segment& sg, int h, const Pass& ps,
                                     PassLds<DK, DV, T, TO>* lds) {
  typedef typename FragFor<T>::type F;
  constexpr int LDK = Rows<DK, T>::LD, LDV = Rows<DV, T>::LD, NS = DV / 64, NQ = DK / 32;
  constexpr int M = kTerms<F, TO>;
  const int w = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const Lane ln = lane_here();
  const int g4 = 4 * ln.g(), c = ln.c(), nc = (sg.len + LC - 1) / LC;
  const bool rev = ps.rev;
  StateOf<DK, DV> S;
  if (ps.start) S.load(ps.start, ps.flip, w, ln); else S.zero();
  Rows<DK, T> q, k;
  Rows<DV, T> v;
  float g = a.per_token ? 0.f : a.g[h];
  auto fetch = [&](int i) __attribute__((always_inline)) {
    const int at = (rev ? nc - 1 - i : i) * LC, m = min(LC, sg.len - at);
    q.load((const T*)ps.q + (int64_t)at * ps.ldq, ps.ldq, m, rev);
    k.load((const T*)ps.k + (int64_t)at * ps.ldk, ps.ldk, m, rev);
    v.load((const T*)ps.v + (int64_t)at * ps.ldv, ps.ldv, m, rev);
    if (a.per_token && w == 0) {
      const int r = min(ln.id, m - 1);
      g = a.g[(sg.t0 + at + (rev ? m - 1 - r : r)) * a.Hv + h];
    }
  };
  // the rows' products with x, of the chunk before: the waves' shares meet in LDS
  auto write_dot = [&](int at, int m) __attribute__((always_inline)) {
    if (ps.dot && w == 1 && ln.id < m)
      ps.dot[at + (rev ? m - 1 - ln.id : ln.id)] =
          (lds->dot[0][ln.id] + lds->dot[1][ln.id]) + (lds->dot[2][ln.id] + lds->dot[3][ln.id]);
    if (ps.dot && threadIdx.x == 0 && m > 0)
      ps.far[at / LC] = (lds->far[0] + lds->far[1]) + (lds->far[2] + lds->far[3]);
  };
  fetch(0);
  int before = 0, mb = 0;
  for (int i = 0; i < nc; ++i) {
    const int at = (rev ? nc - 1 - i : i) * LC, m = min(LC, sg.len - at);
    lds_only_barrier();
    q.store(lds->q, m);
    k.store(lds->k, m);
    v.store(lds->v, m);
    if (w == 0) form_gates(&lds->gt, g, a.per_token, m, rev, ps.s_out, ps.s_in);
    write_dot(before, mb);
    before = at, mb = m;
    if (i + 1 < nc) fetch(i + 1);
    lds_only_barrier();
    // P's row block w, in row form: lane (g, c) has columns 16 J + 4g .. of row 16 w + c
    {
      Pair<F> x[NQ];
#pragma unroll
      for (int s = 0; s < NQ; ++s) x[s] = run_frag<LDK>(lds->q, 16 * w, 32 * s, ln);
      const float hi = lds->gt.hi[16 * w + c], lo = lds->gt.lo[16 * w + c];
      for (int J = 0; J <= (w | 1); ++J) {
        f32x4 p = zero4();
        if (J <= w) {
#pragma unroll
          for (int s = 0; s < NQ; ++s)
            p = Pair<F>::template mma<true>(x[s], run_frag<LDK>(lds->k, 16 * J, 32 * s, ln), p);
          const f32x4 hj = *(const f32x4*)(lds->gt.hi + 16 * J + g4);
          const f32x4 lj = *(const f32x4*)(lds->gt.lo + 16 * J + g4);
#pragma unroll
          for (int u = 0; u < 4; ++u) {
            const float d = __builtin_amdgcn_exp2f((hi - hj[u]) + (lo - lj[u]));
            p[u] = 16 * J + g4 + u <= 16 * w + c ? a.scale * p[u] * d : 0.f;
          }
        }
        T* to = lds->p + p_slot(w, J >> 1) * M * 512;
        if constexpr (M == 1 && sizeof(T) == 4) {
          *(f32x4*)(to + 256 * (J & 1) + 4 * ln.id) = p;
        } else {
          typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));
          float p0 = p[0], p1 = p[1], p2 = p[2], p3 = p[3];
#pragma unroll
          for (int t = 0; t < M; ++t) {
            const u32x2 b{take2(p0, p1), take2(p2, p3)};
            *(u32x2*)(to + t * 512 + 8 * ln.id + 4 * (J & 1)) = b;
          }
        }
      }
    }
    // what comes from the state
    f32x4 o[4][NS];
#pragma unroll
    for (int I = 0; I < 4; ++I)
#pragma unroll
      for (int n = 0; n < NS; ++n) o[I][n] = zero4();
#pragma unroll
    for (int s = 0; s < NQ; ++s) {
      Some<F, M> y[NS];
#pragma unroll
      for (int n = 0; n < NS; ++n) y[n] = some<F, TO>(S.b[2 * s][n], S.b[2 * s + 1][n]);
#pragma unroll
      for (int I = 0; I < 4; ++I) {
        const Pair<F> x = run_frag<LDK>(lds->q, 16 * I, 32 * s, ln);
#pragma unroll
        for (int t = M - 1; t >= 0; --t)
#pragma unroll
          for (int n = 0; n < NS; ++n) o[I][n] = Pair<F>::template mma<true>(x, y[n].t[t], o[I][n]);
      }
    }
#pragma unroll
    for (int I = 0; I < 4; ++I) {
      const float f = lds->gt.out[16 * I + c];
#pragma unroll
      for (int n = 0; n < NS; ++n) o[I][n] *= f;
    }
    // lane (g, c): columns 16 NS w + 4 NS g + 0 .. 4 NS - 1 of row 16 I + c
    const int col = 16 * NS * w + NS * g4;
    auto row_of = [&](int I) { return (int64_t)(at + (rev ? m - 1 - 16 * I - c : 16 * I + c)); };
    RunOf<T, 4 * NS> x[4];
    float far = 0.f;
    if (ps.x) {
#pragma unroll
      for (int I = 0; I < 4; ++I)
        if (16 * I + c < m) {
          x[I] = *(const RunOf<T, 4 * NS>*)((const T*)ps.x + row_of(I) * ps.ldo + col);
#pragma unroll
          for (int n = 0; n < NS; ++n)
#pragma unroll
            for (int u = 0; u < 4; ++u)
              far = __builtin_fmaf((float)x[I][4 * n + u], o[I][n][u], far);
        }
    }
    S.template update<TS>(lds->k, lds->v, &lds->gt, w, ln);
    lds_only_barrier();
    // and from the chunk's tokens
#pragma unroll
    for (int p = 0; p < 2; ++p) {
      Pair<F> y[NS];
#pragma unroll
      for (int n = 0; n < NS; ++n)
        y[n] = down_frag<LDV, 4 * NS>(lds->v, 32 * p, 16 * NS * w + 4 * n, ln);
#pragma unroll
      for (int I = 2 * p; I < 4; ++I) {
        const T* from = lds->p + p_slot(I, p) * M * 512;
#pragma unroll
        for (int t = M - 1; t >= 0; --t) {
          Pair<F> x;
          if constexpr (sizeof(T) == 4)
            x = join(*(const f32x4*)(from + 4 * ln.id), *(const f32x4*)(from + 256 + 4 * ln.id));
          else
            x.v = *(const bf16x8*)(from + t * 512 + 8 * ln.id);
#pragma unroll
          for (int n = 0; n < NS; ++n) o[I][n] = Pair<F>::template mma<true>(x, y[n], o[I][n]);
        }
      }
    }
#pragma unroll
    for (int I = 0; I < 4; ++I) {
      float dot = 0.f;
      if (16 * I + c < m) {
        const int64_t to = row_of(I) * ps.ldo + col;
        if (ps.x) {
#pragma unroll
          for (int n = 0; n < NS; ++n)
#pragma unroll
            for (int u = 0; u < 4; ++u)
              dot = __builtin_fmaf((float)x[I][4 * n + u], o[I][n][u], dot);
        }
#pragma unroll
        for (int n = 0; n < NS; ++n) {
          f32x4 y = o[I][n];
          if (ps.acc && !ps.first) y += *(const f32x4*)(ps.acc + to + 4 * n);
          if (ps.acc && !ps.last) {
            *(f32x4*)(ps.acc + to + 4 * n) = y;
          } else {
            typedef T Out __attribute__((ext_vector_type(4)));
            *(Out*)((T*)ps.out + to + 4 * n) = __builtin_convertvector(y, Out);
          }
        }
      }
      if (ps.x) {
        dot = sum_apart32(sum_apart16(dot));
        if (ln.g() == 0) lds->dot[w][16 * I + c] = dot;
      }
    }
    if (ps.x) {
      far = sum_lanes<64>(far);
      if (ln.id == 0) lds->far[w] = far;
    }
  }
  if (ps.fin) S.store(ps.fin, ps.flip, w, ln);
  if (!ps.x) return;
  lds_only_barrier();
  write_dot(before, mb);
  if (ps.anchor) {  // <S, dS> at the segment's end
    float x = 0.f;
    if (ps.against) {
      StateOf<DK, DV> y;
      y.load(ps.against, ps.flip, w, ln);
#pragma unroll
      for (int m = 0; m < 2 * NQ; ++m)
#pragma unroll
        for (int n = 0; n < NS; ++n)
#pragma unroll
          for (int u = 0; u < 4; ++u) x = __builtin_fmaf(S.b[m][n][u], y.b[m][n][u], x);
      x = sum_lanes<64>(x);
    }
    lds_only_barrier();
    if (ln.id == 0) lds->dot[0][w] = x;
    lds_only_barrier();
    if (threadIdx.x == 0)
      *ps.anchor = (lds->dot[0][0] + lds->dot[0][1]) + (lds->dot[0][2] + lds->dot[0][3]);
  }
}

// sequences without tokens: the state stays what it was
__device__ __forceinline__ void copy_state(const LinArgs& a, int s, const float* from, float* to) {
  int64_t t0, base;
  int len;
  a.q.at(s, t0, base, len);
  if (len > 0) return;
  const int64_t n = (int64_t)a.Hv * a.dk * a.dv, at = (int64_t)s * n;
  for (int64_t e = threadIdx.x * 4; e < n; e += 1024)
    *(f32x4*)(to + at + e) = from ? *(const f32x4*)(from + at + e) : zero4();
}

}  // namespace

template <int DK, int DV, typename T, int TS, int TO>
__global__ __launch_bounds__(256, sizeof(T) == 2 ? 2 : 1) void k_lin_forward(const LinArgs a,
                                                                            uint32_t n) {
  __shared__ __attribute__((aligned(16))) PassLds<DK, DV, T, TO> lds;
  const uint32_t blocks = (n + 7) & ~7u;
  if (blockIdx.x >= blocks) return copy_state(a, (int)(blockIdx.x - blocks), a.S0, a.Sf);
  const uint32_t w = work_item(blockIdx.x, n);
  if (w >= n) return;
  const uint32_t slot = w / (uint32_t)a.Hv;
  const int h = (int)(w - slot * (uint32_t)a.Hv), hk = h / (a.Hv / a.Hk);
  const Segment sg(a.q, slot);
  if (sg.len == 0) return;
  const int64_t size = DK * DV, own = ((int64_t)sg.s * a.Hv + h) * size;
  Pass ps{};
  ps.ldq = ps.ldk = (uint32_t)a.Hk * DK, ps.ldv = ps.ldo = (uint32_t)a.Hv * DV;
  ps.q = (const T*)a.Q + (sg.t0 * a.Hk + hk) * DK;
  ps.k = (const T*)a.K + (sg.t0 * a.Hk + hk) * DK;
  ps.v = (const T*)a.V + (sg.t0 * a.Hv + h) * DV;
  ps.out = (T*)a.O + (sg.t0 * a.Hv + h) * DV;
  ps.start = a.U ? a.U + ((int64_t)slot * a.Hv + h) * size : a.S0 ? a.S0 + own : nullptr;
  ps.fin = a.Sf && sg.j == sg.n - 1 ? a.Sf + own : nullptr;
  ps.s_out = a.scale, ps.s_in = 1.f;
  walk<DK, DV, T, TS, TO>(a, sg, h, ps, &lds);
}

// Three passes: dQ and dK by key heads (the heads of a group one after the other), dV by
// value heads.
template <int DK, int DV, typename T, int TS, int TO>
__global__ __launch_bounds__(256, sizeof(T) == 2 ? 2 : 1) void k_lin_backward(const LinArgs a,
                                                                             uint32_t slots) {
  union Lds {
    PassLds<DV, DK, T, TO> qk;
    PassLds<DK, DV, T, TO> v;
  };
  __shared__ __attribute__((aligned(16))) Lds lds;
  const uint32_t nk = slots * (uint32_t)a.Hk, nv = slots * (uint32_t)a.Hv;
  const uint32_t bk = (2 * nk + 7) & ~7u, bv = (nv + 7) & ~7u;
  const int64_t size = DK * DV;
  if (blockIdx.x >= bk + bv) return copy_state(a, (int)(blockIdx.x - bk - bv), a.dSf, a.dS0);
  const int gr = a.Hv / a.Hk;
  if (blockIdx.x < bk) {
    uint32_t w = work_item(blockIdx.x, 2 * nk);
    if (w >= 2 * nk) return;
    const bool rev = w >= nk;
    if (rev) w -= nk;
    const uint32_t slot = w / (uint32_t)a.Hk;
    const int hk = (int)(w - slot * (uint32_t)a.Hk);
    const Segment sg(a.q, slot);
    if (sg.len == 0) return;
    const int64_t tk = (sg.t0 * a.Hk + hk) * DK;
    for (int u = 0; u < gr; ++u) {
      const int h = hk * gr + u;
      const int64_t tv = (sg.t0 * a.Hv + h) * DV, own = ((int64_t)sg.s * a.Hv + h) * size;
      const int64_t at = ((int64_t)slot * a.Hv + h) * size;
      const int64_t tokens = a.q.cu ? (int64_t)a.q.T : (int64_t)a.q.nseq * a.q.T;
      const float* dS = a.R ? a.R + at : a.dSf ? a.dSf + own : nullptr;
      Pass ps{};
      ps.ldq = ps.ldk = (uint32_t)a.Hv * DV, ps.ldv = ps.ldo = (uint32_t)a.Hk * DK;
      ps.q = (const T*)(rev ? a.V : a.dO) + tv;
      ps.k = (const T*)(rev ? a.dO : a.V) + tv;
      ps.v = (const T*)(rev ? a.Q : a.K) + tk;
      ps.out = (T*)(rev ? a.dK : a.dQ) + tk;
      ps.acc = gr > 1 ? (rev ? a.acc_k : a.acc_q) + tk : nullptr;
      ps.first = u == 0, ps.last = u == gr - 1;
      ps.flip = true, ps.rev = rev;
      if (a.want_dg) {
        ps.x = (const T*)(rev ? a.K : a.Q) + tk;
        ps.dot = (rev ? a.rows_k : a.rows_q) + h * tokens + sg.t0;
        ps.far = (rev ? a.far_k : a.far_q) + ((int64_t)slot * a.Hv + h) * (a.q.seg / LC);
      }
      if (rev) {
        ps.start = dS;
        ps.s_out = 1.f, ps.s_in = a.scale;
      } else {
        ps.start = a.U ? a.U + at : a.S0 ? a.S0 + own : nullptr;
        ps.s_out = a.scale, ps.s_in = 1.f;
        if (a.want_dg) ps.against = dS, ps.anchor = a.anchor + (int64_t)slot * a.Hv + h;
      }
      walk<DV, DK, T, TS, TO>(a, sg, h, ps, &lds.qk);
      lds_only_barrier();
    }
  } else {
    const uint32_t w = work_item(blockIdx.x - bk, nv);
    if (w >= nv) return;
    const uint32_t slot = w / (uint32_t)a.Hv;
    const int h = (int)(w - slot * (uint32_t)a.Hv), hk = h / gr;
    const Segment sg(a.q, slot);
    if (sg.len == 0) return;
    const int64_t tk = (sg.t0 * a.Hk + hk) * DK, tv = (sg.t0 * a.Hv + h) * DV;
    const int64_t own = ((int64_t)sg.s * a.Hv + h) * size;
    Pass ps{};
    ps.ldq = ps.ldk = (uint32_t)a.Hk * DK, ps.ldv = ps.ldo = (uint32_t)a.Hv * DV;
    ps.q = (const T*)a.K + tk, ps.k = (const T*)a.Q + tk, ps.v = (const T*)a.dO + tv;
    ps.out = (T*)a.dV + tv;
    ps.start = a.R ? a.R + ((int64_t)slot * a.Hv + h) * size : a.dSf ? a.dSf + own : nullptr;
    ps.fin = a.dS0 && sg.j == 0 ? a.dS0 + own : nullptr;
    ps.rev = true;
    ps.s_out = 1.f, ps.s_in = a.scale;
    walk<DK, DV, T, TS, TO>(a, sg, h, ps, &lds.v);
  }
}

// ---- the gradient of g: sums over a segment's rows from its end; a wave takes a chunk
__global__ __launch_bounds__(256) void k_lin_decay(const LinArgs a) {
  __shared__ float wave[4];
  const uint32_t slot = blockIdx.x / (uint32_t)a.Hv;
  const int h = (int)(blockIdx.x - slot * (uint32_t)a.Hv);
  const int w = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), l = lane_id();
  const Segment sg(a.q, slot);
  const int64_t at = (int64_t)slot * a.Hv + h;
  const int64_t tokens = a.q.cu ? (int64_t)a.q.T : (int64_t)a.q.nseq * a.q.T;
  const float* rq = a.rows_q + h * tokens + sg.t0;
  const float* rk = a.rows_k + h * tokens + sg.t0;
  const float* fq = a.far_q + at * (a.q.seg / LC);
  const float* fk = a.far_k + at * (a.q.seg / LC);
  const int nc = (sg.len + LC - 1) / LC;
  float all = 0.f;
  for (int c = w; c < nc; c += 4) {
    float z = 0.f;  // <S, dS> at the chunk's end
    for (int i = c + 1 + l; i < nc; i += 64) z += fq[i] - fk[i];
    z = sum_lanes<64>(z) + a.anchor[at];
    // lane l has the l-th token from the chunk's end
    const int m = min(LC, sg.len - c * LC), t = c * LC + m - 1 - l;
    const float d = l < m ? rq[t] - rk[t] : 0.f;
    z += (float)prefix64(d);
    if (l < m) {
      if (a.per_token) a.dg[(sg.t0 + t) * a.Hv + h] = z;
      all += z;
    }
  }
  if (a.per_token) return;
  all = sum_lanes<64>(all);
  if (l == 0) wave[w] = all;
  __syncthreads();
  if (threadIdx.x == 0) a.part[at] = (wave[0] + wave[1]) + (wave[2] + wave[3]);
}

// dg[h] = sum over the segments
__global__ __launch_bounds__(256) void k_lin_decay_sum(const LinArgs a, int64_t slots) {
  __shared__ double s[256];
  const int h = blockIdx.x;
  double x = 0.0;
  for (int64_t i = threadIdx.x; i < slots; i += 256) x += a.part[i * a.Hv + h];
  s[threadIdx.x] = x;
  __syncthreads();
  for (int o = 128; o > 0; o >>= 1) {
    if (threadIdx.x < o) s[threadIdx.x] += s[threadIdx.x + o];
    __syncthreads();
  }
  if (threadIdx.x == 0) a.dg[h] = (float)s[0];
}

int lin_segment(int nseq, int T, int heads, bool packed, bool backward) {
  const int64_t tokens = packed ? (int64_t)T : (int64_t)nseq * T;
  const int whole = (int)((std::min<int64_t>(T, 0x7fffffff - LC) + LC - 1) / LC * LC);
  // about 512 workgroups of work: two a CU
  int64_t seg = tokens * heads / 512 / LC * LC;
  if (seg < 256) seg = 256;
  const int64_t most = backward ? 1024 : 4096;
  if (seg > most) seg = most;
  return seg >= whole ? std::max(whole, LC) : (int)seg;
}

int64_t lin_workspace(LinArgs& a, bool backward, float* ws) {
  const int64_t slots = a.q.slots(), size = (int64_t)a.dk * a.dv;
  const int64_t tokens = a.q.cu ? (int64_t)a.q.T : (int64_t)a.q.nseq * a.q.T;
  const bool many = a.q.seg < a.q.T;
  int64_t n = 0;
  auto take = [&](float*& p, int64_t m) {
    p = ws && m ? ws + n : nullptr;
    n += (m + 3) / 4 * 4;
  };
  take(a.U, many ? slots * a.Hv * size : 0);
  take(a.R, many && backward ? slots * a.Hv * size : 0);
  take(a.dec, many ? slots * a.Hv : 0);
  const bool dg = backward && a.want_dg;
  take(a.rows_q, dg ? a.Hv * tokens : 0);
  take(a.rows_k, dg ? a.Hv * tokens : 0);
  take(a.far_q, dg ? slots * a.Hv * (a.q.seg / LC) : 0);
  take(a.far_k, dg ? slots * a.Hv * (a.q.seg / LC) : 0);
  take(a.anchor, dg ? slots * a.Hv : 0);
  take(a.part, dg && !a.per_token ? slots * a.Hv : 0);
  const bool acc = backward && a.Hv > a.Hk;
  take(a.acc_q, acc ? tokens * a.Hk * a.dk : 0);
  take(a.acc_k, acc ? tokens * a.Hk * a.dk : 0);
  return n;
}

namespace {

hipError_t launch_states(const LinArgs& a, int dtype, bool both, hipStream_t st) {
  const uint32_t n = (uint32_t)(a.q.slots() * a.Hv), grid = (n * (both ? 2 : 1) + 7) & ~7u;
  GDN_DK_SWITCH(a.dk, GDN_DV_SWITCH(a.dv, {
    if (dtype == 0)
      hipLaunchKernelGGL((k_lin_state<DK, DV, float, 1>), dim3(grid), dim3(256), 0, st, a, n, both);
    else
      hipLaunchKernelGGL((k_lin_state<DK, DV, __bf16, 3>), dim3(grid), dim3(256), 0, st, a, n,
                         both);
    if (hipError_t e = hipGetLastError()) return e;
    constexpr int parts = DK * DV / 1024;
    const int64_t heads = std::min<int64_t>((int64_t)a.q.nseq * a.Hv, 16384);
    hipLaunchKernelGGL(k_lin_scan, dim3((unsigned)(heads * parts), both ? 2 : 1), dim3(256), 0, st,
                       a, parts);
    return hipGetLastError();
  }))
  return hipErrorNotSupported;
}

}  // namespace

hipError_t launch_linear_forward(const LinArgs& a, int dtype, hipStream_t st) {
  if (a.U)
    if (hipError_t e = launch_states(a, dtype, false, st)) return e;
  const uint32_t n = a.q.T > 0 ? (uint32_t)(a.q.slots() * a.Hv) : 0;
  const uint32_t grid = ((n + 7) & ~7u) + (a.Sf && (a.q.cu || a.q.T == 0) ? a.q.nseq : 0);
  if (grid == 0) return hipSuccess;
  GDN_DK_SWITCH(a.dk, GDN_DV_SWITCH(a.dv, {
    if (dtype == 0)
      hipLaunchKernelGGL((k_lin_forward<DK, DV, float, 1, 1>), dim3(grid), dim3(256), 0, st, a, n);
    else
      hipLaunchKernelGGL((k_lin_forward<DK, DV, __bf16, 3, 2>), dim3(grid), dim3(256), 0, st, a, n);
    return hipGetLastError();
  }))
  return hipErrorNotSupported;
}

hipError_t launch_linear_backward(const LinArgs& a, int dtype, hipStream_t st) {
  if (a.U)
    if (hipError_t e = launch_states(a, dtype, true, st)) return e;
  const uint32_t slots = a.q.T > 0 ? (uint32_t)a.q.slots() : 0;
  const uint32_t grid = ((2 * slots * a.Hk + 7) & ~7u) + ((slots * a.Hv + 7) & ~7u) +
                        (a.dS0 && (a.q.cu || a.q.T == 0) ? a.q.nseq : 0);
  if (grid > 0) {
    GDN_DK_SWITCH(a.dk, GDN_DV_SWITCH(a.dv, {
      if (dtype == 0)
        hipLaunchKernelGGL((k_lin_backward<DK, DV, float, 1, 1>), dim3(grid), dim3(256), 0, st, a,
                           slots);
      else
        hipLaunchKernelGGL((k_lin_backward<DK, DV, __bf16, 3, 3>), dim3(grid), dim3(256), 0, st,
                           a, slots);
      break;
    }) break;)
    if (hipError_t e = hipGetLastError()) return e;
  }
  if (!a.want_dg) return hipSuccess;
  if (slots > 0) {
    hipLaunchKernelGGL(k_lin_decay, dim3(slots * a.Hv), dim3(256), 0, st, a);
    if (hipError_t e = hipGetLastError()) return e;
  }
  if (!a.per_token) {
    hipLaunchKernelGGL(k_lin_decay_sum, dim3(a.Hv), dim3(256), 0, st, a, (int64_t)slots);
    return hipGetLastError();
  }
  return hipSuccess;
}

}  // namespace gdn
