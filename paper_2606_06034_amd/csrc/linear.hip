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
// before r all of the above holds as it stands.  The gradient of a token's g is
// the sum over what passes the token: pairs of tokens i >= t > j of its chunk, what the state
// that enters the chunk gives tokens i >= t, what tokens j < t give the state that leaves, and
// what passes the chunk:
//   dg_t = sum_{i >= t > j} M_ij + sum_{i >= t} q_i . dQs_i + sum_{j < t} k_j . dKs_j + X,
//   M = ((Q K^T) (.) (scale dO V^T) (.) D), X = e^total <S, dS>, dQs and dKs the states' shares.
// From a chunk to the one before it X + sum q . dQs = X' + sum k . dKs' (the pairs that pass the
// border), so that X is formed once a segment, at its first chunk.  (Sums of q . dQ - k . dK alone, which
// the same pairs cancel in, leave the roundings of all later tokens on a head that has long
// forgotten them.)
//
// A sequence is cut into segments, which workgroups walk chunk by chunk with the state in
// registers.  More than one segment: k_lin_state forms what each adds to the state,
// k_lin_scan carries the states over the segments, k_lin_forward / k_lin_backward walk.
//
// Precision.  bf16 inputs are exact operands of the matrix instructions; fp32 factors
// (states, decayed values, P) enter as sums of three bf16 terms (split.hpp), 2^-24 of each.  (Two
// where a result is in bf16 take 2 to 9 % less time, and are off by several roundings of a
// result whose terms cancel to a thousandth.)  fp32 inputs go to the fp32 matrix instructions.
//
// Bound: a pass's tiles are read once, at 2.8 TB/s; the rest is the serial step of a chunk,
// products of at most 128 x 128 x 64 with the splits between them.  A step takes 4.6 us with
// one workgroup of 256 a CU and 3.8 each with two, 12 with two teams of a gradient.  (8192 tokens,
// 16 heads: states 22 us, their carry 8, walk 54; gradients: states 34, carry 12, dQ 67,
// dK and dV 99, dg 10.)
#include <algorithm>
#include <cmath>

#include "lanes.hpp"
#include "launch.hpp"
#include "layer.hpp"
#include "linear.hpp"
#include "split.hpp"

namespace gdn {

namespace {

// A value that the compiler takes for new at this point.  What a loop derives from it, LDS
// addresses above all, is formed again each time: kept from outside the loop, they were more
// registers than there are and came from scratch memory one after the other.
__device__ __forceinline__ int anew(int x) {
  asm volatile("" : "+v"(x));
  return x;
}

template <typename T> struct FragFor { typedef f32x4 type; };
template <> struct FragFor<__bf16> { typedef bf16x4 type; };

// Blocks of 16 value columns a wave has where a segment's state is formed: eight waves for 128
// columns, as many loads in flight as there can be.  Four walk (eight took as long, 47 and 48 us
// for 16 heads of 8192 tokens in two terms: they take twice the LDS reads of P and leave no room
// for a second workgroup).
constexpr int kStateBlocks = 1;
constexpr int kMostChunks = 16;  // of a segment of the backward pass

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
  float el;                               // e^total
  double sum;                             // of the totals, in units of log 2 (k_lin_state)
};
__device__ __forceinline__ double log_decay(float g) {
  return (double)(g < -1e4f ? -1e4f : g) * kLog2e;
}
// wave-wide: row l of m, `g` its token's (per_token) or the head's; returns the total
// (after: what the rows' values decay by past the chunk, as well)
__device__ __forceinline__ double form_gates(Gates* s, float g, bool per_token, int m, bool rev,
                                             float s_out, float s_in, double after = 0.0) {
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
  s->in[l] = s_in * exp2_of((total - H) + after);
  if (l == 0) s->el = exp2_of(total);
  return total;
}

// A chunk's rows of one head in LDS: D values a row in 16-byte pieces, piece p of row r at
// position p ^ turn(r).  The 16 rows of a run fragment and the 4 x 4 blocks of a transposing
// read both meet 16 different groups of 4 banks (rows padded to 136 values met 2 to 4 times
// the same in the second: half of the LDS cycles were conflicts).
template <int D, typename T>
struct Tile {
  static constexpr int E = 16 / sizeof(T), CPR = D / E;
  static __device__ __forceinline__ int turn(int r) {
    return CPR == 8 ? (r >> 1 & 1) << 2 | (r >> 2 & 3) : (r & 3) << 2 | (r >> 2 & 3);
  }
  static __device__ __forceinline__ int at(int r, int c) {
    return r * D + ((c / E) ^ turn(r)) * E + c % E;
  }
};

// The same on the way from memory, NT threads: thread t has the pieces of one column of rows
// t / CPR, and NT / CPR further each.
template <int D, int NT, typename T>
struct Rows {
  typedef Tile<D, T> L;
  static constexpr int E = L::E, CPR = L::CPR, N = LC * CPR / NT, R = NT / CPR;
  typedef T Vec __attribute__((ext_vector_type(E)));
  Vec v[N];
  // t: the thread; p: the chunk's first token, ld values a token; rows past m repeat one of its own
  template <bool REV>
  __device__ __forceinline__ void load(const T* __restrict__ p, uint32_t ld, int m, int t) {
    const uint32_t r0 = (uint32_t)t / CPR, c = (uint32_t)t % CPR * E;
    if (m == LC) {  // one offset a lane, the rest is the wave's
      const uint32_t off = ((REV ? R - 1 - r0 : r0) * ld + c) * sizeof(T);
#pragma unroll
      for (int i = 0; i < N; ++i) {
        const T* pi = p + (int64_t)((REV ? N - 1 - i : i) * R) * ld;
        v[i] = *(const Vec*)((const char*)pi + off);
      }
    } else {
#pragma unroll
      for (int i = 0; i < N; ++i) {
        const int r = min((int)r0 + R * i, m - 1);
        v[i] = *(const Vec*)(p + ((uint32_t)(REV ? m - 1 - r : r) * ld + c));
      }
    }
  }
  __device__ __forceinline__ void store(T* s, int m, int t) const {
    const int r0 = (uint32_t)t / CPR, c = (uint32_t)t % CPR * E;
    auto to = [&](int i) {  // (rows 16 apart are turned alike)
      return R % 16 == 0 ? s + L::at(r0, c) + i * R * D : s + L::at(r0 + R * i, c);
    };
    if (m == LC) {
#pragma unroll
      for (int i = 0; i < N; ++i) *(Vec*)to(i) = v[i];
    } else {
#pragma unroll
      for (int i = 0; i < N; ++i) *(Vec*)to(i) = r0 + R * i < m ? v[i] : Vec{};
    }
  }
};

// Fragments of a tile.  Along a row: slot s of lane (g, c) is value 8g + s of the run at c0 of
// row r0 + c.  Down the rows: slot s is row r0 + 16 (s / 4) + 4g + s % 4 of column c0 +
// GS (c / 4) + c % 4.
template <int D>
__device__ __forceinline__ Pair<bf16x4> run_frag(const __bf16* s, int r0, int c0, Lane ln) {
  return Pair<bf16x4>{*(const bf16x8*)(s + Tile<D, __bf16>::at(ln.c(), c0 + 8 * ln.g()) + r0 * D)};
}
template <int D>
__device__ __forceinline__ Pair<f32x4> run_frag(const float* s, int r0, int c0, Lane ln) {
  typedef Tile<D, float> L;
  const int c = c0 + 8 * ln.g();
  return join(*(const f32x4*)(s + L::at(ln.c(), c) + r0 * D),
              *(const f32x4*)(s + L::at(ln.c(), c + 4) + r0 * D));
}
template <int D, int GS>
__device__ __forceinline__ Pair<bf16x4> down_frag(const __bf16* s, int r0, int c0, Lane ln) {
  const __bf16* p = s + Tile<D, __bf16>::at(4 * ln.g() + (ln.c() >> 2), c0 + GS * (ln.c() & 3)) +
                    r0 * D;
  return join(read_transposed(p), read_transposed(p + 16 * D));
}
template <int D, int GS>
__device__ __forceinline__ Pair<f32x4> down_frag(const float* s, int r0, int c0, Lane ln) {
  f32x4 a, b;
#pragma unroll
  for (int v = 0; v < 4; ++v) {
    const float* p =
        s + Tile<D, float>::at(4 * ln.g() + v, c0 + GS * (ln.c() >> 2) + (ln.c() & 3)) + r0 * D;
    a[v] = p[0], b[v] = p[16 * D];
  }
  return join(a, b);
}

// 8 values of a row
template <typename F>
__device__ __forceinline__ Pair<F> load_run8(const __bf16* p) {
  return Pair<F>{*(const bf16x8*)p};
}
template <typename F>
__device__ __forceinline__ Pair<F> load_run8(const float* p) {
  return Pair<F>{*(const f32x4*)p, *(const f32x4*)(p + 4)};
}

// A wave's part of a [DK, DV] state: all rows, NS blocks of 16 columns.  Block m = 2q + h,
// block row 4g + v holds state row 32q + 8g + 4h + v, so that two blocks are the pair that
// meets a run of 8 values of a row; column c of block n of wave w is 16 NS w + 4 NS (c / 4) + 4n +
// c % 4, so that a row-form result has 4 NS neighbouring columns a lane.
template <int DK, int DV, int NS>
struct StateOf {
  static constexpr int NQ = DK / 32;
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
      for (int n = 0; n < NS; ++n) b[m][n] = block(p, flip, m, n, w, ln);
  }
  static __device__ __forceinline__ f32x4 block(const float* p, bool flip, int m, int n, int w,
                                                Lane ln) {
    const int r = row(m, ln), c = col(n, w, ln);
    if (flip) return *(const f32x4*)(p + c * DK + r);
    return f32x4{p[r * DV + c], p[(r + 1) * DV + c], p[(r + 2) * DV + c], p[(r + 3) * DV + c]};
  }
  __device__ __forceinline__ void store(float* p, int w, Lane ln) const {
#pragma unroll
    for (int m = 0; m < 2 * NQ; ++m)
#pragma unroll
      for (int n = 0; n < NS; ++n) {
        const int r = row(m, ln), c = col(n, w, ln);
#pragma unroll
        for (int v = 0; v < 4; ++v) p[(r + v) * DV + c] = b[m][n][v];
      }
  }
  __device__ __forceinline__ void decay(float el) {
#pragma unroll
    for (int m = 0; m < 2 * NQ; ++m)
#pragma unroll
      for (int n = 0; n < NS; ++n) b[m][n] *= el;
  }
  // S <- S + (diag(in) K)^T V of the chunk in LDS, the factor on V's rows
  template <typename T>
  __device__ __forceinline__ void update(const T* sK, const T* sV, const Gates* gt, int w,
                                         Lane ln) {
    typedef typename FragFor<T>::type F;
#pragma unroll
    for (int p = 0; p < 2; ++p) {
      const f32x4 wl = *(const f32x4*)(gt->in + 32 * p + 4 * ln.g());
      const f32x4 wh = *(const f32x4*)(gt->in + 32 * p + 16 + 4 * ln.g());
      Terms<F> y[NS];
#pragma unroll
      for (int n = 0; n < NS; ++n) {
        const Pair<F> x = down_frag<DV, 4 * NS>(sV, 32 * p, 16 * NS * w + 4 * n, ln);
        y[n] = split<F>(x.lo() * wl, x.hi() * wh);
      }
#pragma unroll
      for (int m0 = 0; m0 < 2 * NQ; m0 += 2) {  // 2 NS sums side by side
        Pair<F> k[2];
#pragma unroll
        for (int m = 0; m < 2; ++m)
          k[m] = down_frag<DK, 8>(sK, 32 * p, 16 * m0 + 4 * m, ln);
#pragma unroll
        for (int i = TermsOf<F>::N - 1; i >= 0; --i)
#pragma unroll
          for (int m = 0; m < 2; ++m)
#pragma unroll
            for (int n = 0; n < NS; ++n)
              b[m0 + m][n] = Pair<F>::template mma<false>(k[m], y[n].t[i], b[m0 + m][n]);
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

// Its chunks in the order of the walk
struct Chunks {
  int n, len;
  bool rev;
  __device__ Chunks(const Segment& sg, bool r) : n((sg.len + LC - 1) / LC), len(sg.len), rev(r) {}
  __device__ __forceinline__ int at(int i) const { return (rev ? n - 1 - i : i) * LC; }
  __device__ __forceinline__ int size(int i) const { return min(LC, len - at(i)); }
  // token of row r
  __device__ __forceinline__ int token(int i, int r) const {
    return at(i) + (rev ? size(i) - 1 - r : r);
  }
};

// The gates of a walk's chunks, formed by one wave a chunk ahead (two tables in turn): on the
// way of all waves they were 60 dependent instructions, half of them in 64 bits.
struct GateStream {
  const LinArgs& a;
  const Chunks& ch;
  const float* g;  // the segment's first token's
  float now;
  bool mine;
  float s_out, s_in;
  __device__ GateStream(const LinArgs& a_, const Segment& sg, const Chunks& c, int h, bool m, float so,
                        float si)
      : a(a_), ch(c), g(a_.g + (a_.per_token ? sg.t0 * a_.Hv + h : h)), mine(m), s_out(so), s_in(si) {
    now = mine && !a.per_token ? *g : 0.f;
    fetch(0);
  }
  __device__ __forceinline__ void fetch(int i) {
    if (mine && a.per_token && i < ch.n)
      now = g[(int64_t)ch.token(i, min(lane_id(), ch.size(i) - 1)) * a.Hv];
  }
  // those of chunk i, at the buffer that chunk i - 2 has left
  __device__ __forceinline__ void form(Gates* two, int i) {
    if (!mine || i >= ch.n) return;
    form_gates(two + (i & 1), now, a.per_token, ch.size(i), ch.rev, s_out, s_in);
    fetch(i + 1);
  }
};

// work item of a workgroup: neighbours on one XCD (workgroups go round the 8 in turn)
__device__ __forceinline__ uint32_t work_item(uint32_t b, uint32_t n) {
  return (b & 7) * ((n + 7) >> 3) + (b >> 3);
}

// ---- what a segment adds to the state
template <int DK, int DV, int NS, typename T, bool REV>
__device__ __forceinline__ void add_of_segment(const LinArgs& a, const Segment& sg, uint32_t slot,
                                               int h, T* sK, T* sV, Gates* gt) {
  constexpr bool rev = REV;
  const int gr = a.Hv / a.Hk;
  const T* K = (const T*)(rev ? a.Q : a.K) + (sg.t0 * a.Hk + h / gr) * DK;
  const T* V = (const T*)(rev ? a.dO : a.V) + (sg.t0 * a.Hv + h) * DV;
  const uint32_t ldk = (uint32_t)a.Hk * DK, ldv = (uint32_t)a.Hv * DV;
  const int w = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const Lane ln = lane_here();
  constexpr int NT = 4 * DV / NS;
  const Chunks ch(sg, rev);
  StateOf<DK, DV, NS> S;
  S.zero();
  Rows<DK, NT, T> k;
  Rows<DV, NT, T> v;
  auto fetch = [&](int i) __attribute__((always_inline)) {
    const int at = ch.at(i), m = ch.size(i);
    k.template load<REV>(K + (int64_t)at * ldk, ldk, m, threadIdx.x);
    v.template load<REV>(V + (int64_t)at * ldv, ldv, m, threadIdx.x);
  };
  // From the last chunk to the first, each decayed past those after it, so that nothing is
  // scaled again; and no further than to where the decay is 0 as a factor in fp32 (2^-160:
  // below 2^-149 there is none).
  constexpr double kNothing = -160.0;
  double total = 0.0;  // of the chunks so far: the first wave's
  auto gates = [&](int i, float g) __attribute__((always_inline)) {
    if (w != 0) return;
    total += form_gates(gt + (i & 1), g, a.per_token, ch.size(i), rev, 1.f, rev ? a.scale : 1.f,
                        total);
    if (ln.id == 0) gt[i & 1].sum = total;
  };
  auto decay_of = [&](int i) __attribute__((always_inline)) {
    if (i < 0 || w != 0) return 0.f;
    return a.per_token
               ? a.g[(sg.t0 + ch.token(i, min(ln.id, ch.size(i) - 1))) * (int64_t)a.Hv + h]
               : a.g[h];
  };
  int i = ch.n - 1;
  float g = decay_of(i);
  fetch(i);
  gates(i, g);
  g = decay_of(i - 1);
  for (;; --i) {
    lds_only_barrier();
    const bool more = i > 0 && !(gt[i & 1].sum < kNothing);
    k.store(sK, ch.size(i), threadIdx.x);
    v.store(sV, ch.size(i), threadIdx.x);
    if (more) fetch(i - 1);
    lds_only_barrier();
    if (more) {
      gates(i - 1, g);
      g = decay_of(i - 2);
    }
    S.update(sK, sV, gt + (i & 1), w, ln);
    if (!more) break;
  }
  for (; w == 0 && i > 0; --i) {  // (the decay over all of the segment)
    const float x = decay_of(i - 1);
    total += a.per_token ? lane63(prefix64(ln.id < ch.size(i - 1) ? log_decay(x) : 0.0))
                         : log_decay(x) * ch.size(i - 1);
  }
  float* to = (rev ? a.R : a.U) + ((int64_t)slot * a.Hv + h) * DK * DV;
  S.store(to, w, ln);
  if (threadIdx.x == 0 && (!rev || sg.j == sg.n - 1))  // (once for each segment)
    a.dec[(int64_t)slot * a.Hv + h] = exp2_of(total);
}

}  // namespace

// `both`: the gradients' states too, in the second half of the work items
template <int DK, int DV, int NS, typename T>
__global__ __launch_bounds__(4 * DV / NS) void k_lin_state(const LinArgs a, uint32_t n, bool both) {
  __shared__ __attribute__((aligned(16))) T sK[LC * DK], sV[LC * DV];
  __shared__ __attribute__((aligned(16))) Gates gt[2];
  uint32_t w = work_item(blockIdx.x, n * (both ? 2 : 1));
  if (w >= n * (both ? 2 : 1)) return;
  const bool rev = w >= n;
  if (rev) w -= n;
  const uint32_t slot = w / (uint32_t)a.Hv;
  const int h = (int)(w - slot * (uint32_t)a.Hv);
  const Segment sg(a.q, slot);
  // (the last segment's share ends in S_final, the first one's in dS0: the walks form those)
  if (sg.len == 0 || (rev ? sg.j == 0 : sg.j == sg.n - 1)) return;
  if (rev)
    add_of_segment<DK, DV, NS, T, true>(a, sg, slot, h, sK, sV, gt);
  else
    add_of_segment<DK, DV, NS, T, false>(a, sg, slot, h, sK, sV, gt);
}

// The states carried over the segments of each sequence, in place: U from what a segment
// adds to the state that enters it, R to the gradient of the state that leaves it.  Bound: HBM
// where there are many (4 x 8192 tokens of 32 heads, both: 246 MB in 41 us), else the chain of
// loads, eight asked for ahead: 22 us for 16384 packed tokens of 16 heads in segments of 512, 28
// with sixteen (34 in segments of 256); 7.5 either way for 8192 in one.
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
    constexpr int A = 8;  // asked for ahead
    for (int i0 = 0; i0 < n; i0 += A) {
      f32x4 x[A];
      float f[A];
#pragma unroll
      for (int u = 0; u < A; ++u) {
        const int i = i0 + u, j = rev ? n - 1 - i : i;
        if (i + 1 < n) {
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

// One pass along a segment for one value head.
struct Pass {
  const void *q, *k, *v;        // its tiles in LDS
  const void* x;                // rows for the gradient of g, in memory or a tile
  uint32_t ldo;                 // values a token of x and of the result
  void* out;
  float* acc;                   // sums of a group's heads (null: one head, or two side by side)
  bool first, last;             // of the group
  float* rows;                  // x's products of each token, at the segment's first
  const float* start;           // the state that enters (or null: zeros)
  float* fin;                   // the state that leaves (or null)
  const float* against;         // dK: the state that enters (or null: zeros)
  float* anchor;                // dK: X of the segment's first chunk
};

// What a pass forms, and how.
enum Kind { kO, kDQ, kDK, kDV };
template <Kind P> constexpr bool kReversed = P == kDK || P == kDV;
template <Kind P> constexpr bool kFlipped = P == kDQ || P == kDK;  // the state, in memory

// What the waves of a pass share, beside its tiles.
template <int NW, typename T>
struct TeamLds {
  T p[6 * TermsOf<typename FragFor<T>::type>::N * 512];
  float far[NW][LC];             // the waves' shares of x . (what came from the state)
  float row[4][LC], col[4][LC];  // sums of M's blocks (I, J): along rows at J, down columns at I
  Gates gt[2];
  double part[NW];
};

// The tiles of a workgroup, from where they come to LDS, and the passes that read them.
template <int D, int NT, typename T>
struct Source {
  const T* p;
  uint32_t ld;
  T* s;
  Rows<D, NT, T> r;
  __device__ Source(const T* from, int heads, T* to) : p(from), ld((uint32_t)heads * D), s(to) {}
  template <bool REV> __device__ __forceinline__ void fetch(int at, int m, int t) {
    r.template load<REV>(p + (int64_t)at * ld, ld, m, t);
  }
  __device__ __forceinline__ void store(int m, int t) const { r.store(s, m, t); }
};

// P's fragments of row block I: pair p of column blocks
__host__ __device__ constexpr int p_slot(int I, int p) { return (I == 3 ? 4 : I) + p; }

template <typename T, int N> struct RunType { typedef T type __attribute__((ext_vector_type(N))); };
template <typename T, int N> using RunOf = typename RunType<T, N>::type;

// DG: with the rows that the gradient of g takes (of dQ and dK).  A team of NW waves walks;
// two teams of a workgroup walk side by side on tiles that all of them bring, with the same
// barriers.  other: what a second team gives a first one to add to its result (null: none).
// XS: x is a tile (with dK), else rows in memory.
template <int DK, int DV, int NS, typename T, Kind P, bool DG, bool XS, typename Tiles>
__device__ __forceinline__ void walk(const LinArgs& a, const Segment& sg, int h, const Pass& ps,
                                     Tiles& tiles, TeamLds<DV / 16 / NS, T>* lds,
                                     float* other = nullptr) {
  typedef typename FragFor<T>::type F;
  constexpr int NQ = DK / 32, NW = DV / 16 / NS, N = TermsOf<F>::N;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), w = wave % NW;
  const Lane ln = lane_here();
  constexpr bool rev = kReversed<P>, flip = kFlipped<P>;
  constexpr bool far_rows = DG && flip, pairs = DG && P == kDK;
  const Chunks ch(sg, rev);
  StateOf<DK, DV, NS> S;
  if (ps.start) S.load(ps.start, flip, w, ln); else S.zero();
  const T *sq = (const T*)ps.q, *sk = (const T*)ps.k, *sv = (const T*)ps.v;
  // what the gradient of g takes of a chunk: the waves' shares meet in LDS
  auto write_rows = [&](int i) __attribute__((always_inline)) {
    if (!far_rows || w != 3 || i < 0 || ln.id >= ch.size(i)) return;
    float f = 0.f;
#pragma unroll
    for (int u = 0; u < NW; ++u) f += lds->far[u][ln.id];
    if (pairs) {
      float e = 0.f;
#pragma unroll
      for (int u = 0; u < 4; ++u) {
        if (u <= ln.id >> 4) e += lds->row[u][ln.id];
        if (u >= ln.id >> 4) e -= lds->col[u][ln.id];
      }
      f += e;
    }
    ps.rows[ch.token(i, ln.id)] = f;
  };
  GateStream gates(a, sg, ch, h, w == 2, rev ? 1.f : a.scale, rev ? a.scale : 1.f);
  tiles.template fetch<rev>(ch.at(0), ch.size(0), threadIdx.x);
  gates.form(lds->gt, 0);
  // P's blocks above the diagonal that share a pair with one on it
  if (w < 2) {
    T* to = lds->p + p_slot(2 * w, w) * N * 512;
#pragma unroll
    for (int t = 0; t < N; ++t) {
      if constexpr (sizeof(T) == 4)
        *(f32x4*)(to + 256 + 4 * ln.id) = zero4();
      else
        *(uint64_t*)(to + t * 512 + 8 * ln.id + 4) = 0;
    }
  }
  for (int i = 0; i < ch.n; ++i) {
    const Lane ln{anew(lane_id())};
    const int g4 = 4 * ln.g(), c = ln.c();
    const int at = ch.at(i), m = ch.size(i);
    const bool end = i == ch.n - 1;
    const Gates* gt = lds->gt + (i & 1);
    lds_only_barrier();
    tiles.store(m, anew(threadIdx.x));
    write_rows(i - 1);
    lds_only_barrier();
    if (pairs && end) {  // (in 64 bits: dk dv products of any sign)
      double x = 0.0;
      if (ps.against) {
#pragma unroll
        for (int u = 0; u < 2 * NQ; ++u)
#pragma unroll
          for (int n = 0; n < NS; ++n) {
            const f32x4 y = StateOf<DK, DV, NS>::block(ps.against, flip, u, n, w, ln);
#pragma unroll
            for (int e = 0; e < 4; ++e) x = __builtin_fma((double)S.b[u][n][e], (double)y[e], x);
          }
        x = lane63(prefix64(x));
      }
      if (ln.id == 0) lds->part[w] = x;
    }
    // P's blocks in row form: lane (g, c) has columns 16 J + 4g .. of row 16 I + c; two of them
    // at a time
    auto products = [&](int I, int J) __attribute__((always_inline)) {
      f32x4 p0 = zero4(), p1 = zero4();
#pragma unroll
      for (int s = 0; s < NQ; s += 2) {
        p0 = Pair<F>::template mma<true>(run_frag<DK>(sq, 16 * I, 32 * s, ln),
                                         run_frag<DK>(sk, 16 * J, 32 * s, ln), p0);
        p1 = Pair<F>::template mma<true>(run_frag<DK>(sq, 16 * I, 32 * s + 32, ln),
                                         run_frag<DK>(sk, 16 * J, 32 * s + 32, ln), p1);
      }
      return p0 + p1;
    };
    // X V^T, for M
    auto more_products = [&](int I, int J) __attribute__((always_inline)) {
      f32x4 p0 = zero4(), p1 = zero4();
#pragma unroll
      for (int s = 0; s < DV / 32; s += 2) {
        Pair<F> x0, x1;
        if constexpr (XS) {
          x0 = run_frag<DV>((const T*)ps.x, 16 * I, 32 * s, ln);
          x1 = run_frag<DV>((const T*)ps.x, 16 * I, 32 * s + 32, ln);
        } else {
          const T* xp = (const T*)ps.x + (int64_t)ch.token(i, min(16 * I + c, m - 1)) * ps.ldo +
                        32 * s + 2 * g4;
          x0 = load_run8<F>(xp), x1 = load_run8<F>(xp + 32);
        }
        p0 = Pair<F>::template mma<true>(x0, run_frag<DV>(sv, 16 * J, 32 * s, ln), p0);
        p1 = Pair<F>::template mma<true>(x1, run_frag<DV>(sv, 16 * J, 32 * s + 32, ln), p1);
      }
      return p0 + p1;
    };
    auto finish = [&](f32x4 p, f32x4 y, int I, int J) __attribute__((always_inline)) {
      const int r = 16 * I + c;
      const float hi = gt->hi[r], lo = gt->lo[r];
      const f32x4 hj = *(const f32x4*)(gt->hi + 16 * J + g4);
      const f32x4 lj = *(const f32x4*)(gt->lo + 16 * J + g4);
#pragma unroll
      for (int u = 0; u < 4; ++u) {
        const float d = __builtin_amdgcn_exp2f((hi - hj[u]) + (lo - lj[u]));
        p[u] = 16 * J + g4 + u <= r ? a.scale * p[u] * d : 0.f;
      }
      T* to = lds->p + p_slot(I, J >> 1) * N * 512;
      if constexpr (sizeof(T) == 4) {
        *(f32x4*)(to + 256 * (J & 1) + 4 * ln.id) = p;
      } else {
        typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));
        float p0 = p[0], p1 = p[1], p2 = p[2], p3 = p[3];
#pragma unroll
        for (int t = 0; t < N; ++t) {
          const uint32_t x = take2(p0, p1), z = take2(p2, p3);
          *(u32x2*)(to + t * 512 + 8 * ln.id + 4 * (J & 1)) = u32x2{x, z};
        }
      }
      if constexpr (pairs) {  // M, of rows below the diagonal
        float sum = 0.f;
#pragma unroll
        for (int u = 0; u < 4; ++u) {
          y[u] = 16 * J + g4 + u < r && r < m ? y[u] * p[u] : 0.f;
          sum += y[u];
          y[u] = sum16(y[u]);
        }
        sum = sum_apart32(sum_apart16(sum));
        if (ln.g() == 0) lds->row[J][r] = sum;
        if (c == 0) *(f32x4*)(lds->col[I] + 16 * J + g4) = y;
      }
    };
    auto row_of = [](int b) { return b < 1 ? 0 : b < 3 ? 1 : b < 6 ? 2 : 3; };
    static_assert(NW == 4, "two of the ten blocks a wave, and two over");
    {
      const int b1 = w + NW;
      const int I0 = row_of(w), J0 = w - I0 * (I0 + 1) / 2;
      const int I1 = row_of(b1), J1 = b1 - I1 * (I1 + 1) / 2;
      const f32x4 p0 = products(I0, J0), p1 = products(I1, J1);
      f32x4 y0 = zero4(), y1 = zero4();
      if constexpr (pairs) y0 = more_products(I0, J0), y1 = more_products(I1, J1);
      finish(p0, y0, I0, J0);
      finish(p1, y1, I1, J1);
      if (w < 2) {
        const int J = w + 2;  // blocks 8 and 9
        f32x4 y = zero4();
        const f32x4 p = products(3, J);
        if constexpr (pairs) y = more_products(3, J);
        finish(p, y, 3, J);
      }
    }
    // rows of x at the results' places
    RunOf<T, 4 * NS> xr[4];
    if constexpr (far_rows && !XS)
#pragma unroll
      for (int I = 0; I < 4; ++I) {
        const T* xc = (const T*)ps.x + (int64_t)at * ps.ldo + 16 * NS * w;
        const int r = min(16 * I + c, m - 1);
        const uint32_t off = (uint32_t)(rev ? m - 1 - r : r) * ps.ldo + NS * g4;
        xr[I] = *(const RunOf<T, 4 * NS>*)((const char*)xc + off * (uint32_t)sizeof(T));
      }
    gates.form(lds->gt, i + 1);
    // what comes from the state
    f32x4 o[4][NS];
#pragma unroll
    for (int I = 0; I < 4; ++I)
#pragma unroll
      for (int n = 0; n < NS; ++n) o[I][n] = zero4();
#pragma unroll
    for (int s = 0; s < NQ; ++s) {
      Terms<F> y[NS];
#pragma unroll
      for (int n = 0; n < NS; ++n) y[n] = split<F>(S.b[2 * s][n], S.b[2 * s + 1][n]);
#pragma unroll
      for (int I0 = 0; I0 < 4; I0 += 2) {
        Pair<F> x[2];
#pragma unroll
        for (int I = 0; I < 2; ++I) x[I] = run_frag<DK>(sq, 16 * (I0 + I), 32 * s, ln);
#pragma unroll
        for (int t = N - 1; t >= 0; --t)
#pragma unroll
          for (int I = 0; I < 2; ++I)
#pragma unroll
            for (int n = 0; n < NS; ++n)
              o[I0 + I][n] = Pair<F>::template mma<true>(x[I], y[n].t[t], o[I0 + I][n]);
      }
    }
    // lane (g, c): columns 16 NS w + NS g4 .. of row 16 I + c; one offset a lane
    const uint32_t place = (uint32_t)(rev ? 15 - c : c) * ps.ldo + NS * g4;
    auto block = [&](int I) {
      return ((int64_t)at + (rev ? m - 16 - 16 * I : 16 * I)) * ps.ldo + 16 * NS * w;
    };
#pragma unroll
    for (int I = 0; I < 4; ++I) {
      const float f = gt->out[16 * I + c];
#pragma unroll
      for (int n = 0; n < NS; ++n) o[I][n] *= f;
    }
    if constexpr (far_rows)
#pragma unroll
      for (int I = 0; I < 4; ++I) {
        if constexpr (XS)
          xr[I] = *(const RunOf<T, 4 * NS>*)((const T*)ps.x + 16 * I * DV +
                                             Tile<DV, T>::at(c, 16 * NS * w + NS * g4));
        float far = 0.f;
#pragma unroll
        for (int n = 0; n < NS; ++n)
#pragma unroll
          for (int u = 0; u < 4; ++u)
            far = __builtin_fmaf((float)xr[I][4 * n + u], o[I][n][u], far);
        far = sum_apart32(sum_apart16(far));
        if (ln.g() == 0) lds->far[w][16 * I + c] = far;
      }
    if (!end) tiles.template fetch<rev>(ch.at(i + 1), ch.size(i + 1), anew(threadIdx.x));
    S.decay(gt->el);
    S.update(sk, sv, gt, w, ln);
    lds_only_barrier();
    if (pairs && end && w == 0 && ln.id == 0) {
      double x = 0.0;
#pragma unroll
      for (int u = 0; u < NW; ++u) x += lds->part[u];
      *ps.anchor = (float)(gt->el * x);
    }
    // and from the chunk's tokens
#pragma unroll
    for (int p = 0; p < 2; ++p) {
      Pair<F> y[NS];
#pragma unroll
      for (int n = 0; n < NS; ++n)
        y[n] = down_frag<DV, 4 * NS>(sv, 32 * p, 16 * NS * w + 4 * n, ln);
#pragma unroll
      for (int t = N - 1; t >= 0; --t)
#pragma unroll
        for (int I = 2 * p; I < 4; ++I) {
          const T* from = lds->p + (p_slot(I, p) * N + t) * 512;
          Pair<F> x;
          if constexpr (sizeof(T) == 4)
            x = join(*(const f32x4*)(from + 4 * ln.id), *(const f32x4*)(from + 256 + 4 * ln.id));
          else
            x.v = *(const bf16x8*)(from + 8 * ln.id);
#pragma unroll
          for (int n = 0; n < NS; ++n) o[I][n] = Pair<F>::template mma<true>(x, y[n], o[I][n]);
        }
    }
    if (other) {
      if (wave >= NW)
#pragma unroll
        for (int I = 0; I < 4; ++I)
#pragma unroll
          for (int n = 0; n < NS; ++n)
            *(f32x4*)(other + (((w * 4 + I) * NS + n) * 64 + ln.id) * 4) = o[I][n];
      lds_only_barrier();
      if (wave >= NW) continue;
#pragma unroll
      for (int I = 0; I < 4; ++I)
#pragma unroll
        for (int n = 0; n < NS; ++n)
          o[I][n] += *(const f32x4*)(other + (((w * 4 + I) * NS + n) * 64 + ln.id) * 4);
    }
    typedef T Out __attribute__((ext_vector_type(4)));
#pragma unroll
    for (int I = 0; I < 4; ++I)
      if (16 * I + c < m)
#pragma unroll
        for (int n = 0; n < NS; ++n) {
          f32x4 y = o[I][n];
          float* acc = (float*)((char*)(ps.acc + block(I)) + place * 4) + 4 * n;
          if (flip && ps.acc && !ps.first) y += *(const f32x4*)acc;
          if (flip && ps.acc && !ps.last)
            *(f32x4*)acc = y;
          else
            *(Out*)((T*)((char*)((T*)ps.out + block(I)) + place * (uint32_t)sizeof(T)) + 4 * n) =
                __builtin_convertvector(y, Out);
        }
  }
  if (!flip && ps.fin) S.store(ps.fin, w, ln);
  if (!far_rows) return;
  lds_only_barrier();
  write_rows(ch.n - 1);
}

// The tiles of one pass.
template <int DK, int DV, int NT, typename T>
struct PassTiles {
  Source<DK, NT, T> q, k;
  Source<DV, NT, T> v;
  template <bool REV> __device__ __forceinline__ void fetch(int at, int m, int t) {
    q.template fetch<REV>(at, m, t);
    k.template fetch<REV>(at, m, t);
    v.template fetch<REV>(at, m, t);
  }
  __device__ __forceinline__ void store(int m, int t) const {
    q.store(m, t), k.store(m, t), v.store(m, t);
  }
};
// Two of one kind each: of DA and of DB values a row.
template <int DA, int DB, int NT, typename T>
struct TwoAndTwo {
  Source<DA, NT, T> a0, a1;
  Source<DB, NT, T> b0, b1;
  template <bool REV> __device__ __forceinline__ void fetch(int at, int m, int t) {
    a0.template fetch<REV>(at, m, t), a1.template fetch<REV>(at, m, t);
    b0.template fetch<REV>(at, m, t), b1.template fetch<REV>(at, m, t);
  }
  __device__ __forceinline__ void store(int m, int t) const {
    a0.store(m, t), a1.store(m, t), b0.store(m, t), b1.store(m, t);
  }
};
// Those of dQ or dK of two heads, MORE: with x.
template <int DA, int DB, int NT, typename T, bool MORE>
struct FourAndMore {
  Source<DA, NT, T> a0, a1, a2, a3;
  Source<DB, NT, T> b0, b1;
  template <bool REV> __device__ __forceinline__ void fetch(int at, int m, int t) {
    a0.template fetch<REV>(at, m, t), a1.template fetch<REV>(at, m, t);
    a2.template fetch<REV>(at, m, t), a3.template fetch<REV>(at, m, t);
    b0.template fetch<REV>(at, m, t);
    if (MORE) b1.template fetch<REV>(at, m, t);
  }
  __device__ __forceinline__ void store(int m, int t) const {
    a0.store(m, t), a1.store(m, t), a2.store(m, t), a3.store(m, t), b0.store(m, t);
    if (MORE) b1.store(m, t);
  }
};

// sequences without tokens: the state stays what it was
__device__ __forceinline__ void copy_state(const LinArgs& a, int s, const float* from, float* to) {
  int64_t t0, base;
  int len;
  a.q.at(s, t0, base, len);
  if (len > 0) return;
  const int64_t n = (int64_t)a.Hv * a.dk * a.dv, at = (int64_t)s * n;
  for (int64_t e = threadIdx.x * 4; e < n; e += 4 * blockDim.x)
    *(f32x4*)(to + at + e) = from ? *(const f32x4*)(from + at + e) : zero4();
}

}  // namespace

// workgroups a CU, of a wave a SIMD each
template <typename T> constexpr int kGroups = sizeof(T) == 2 ? 2 : 1;

template <int DK, int DV, typename T>
__global__ __launch_bounds__(256, kGroups<T>) void k_lin_forward(const LinArgs a, uint32_t n) {
  constexpr int NS = DV / 64, NT = 256;
  __shared__ __attribute__((aligned(16))) T sq[LC * DK], sk[LC * DK], sv[LC * DV];
  __shared__ __attribute__((aligned(16))) TeamLds<DV / 16 / NS, T> lds;
  const uint32_t blocks = (n + 7) & ~7u;
  if (blockIdx.x >= blocks) return copy_state(a, (int)(blockIdx.x - blocks), a.S0, a.Sf);
  const uint32_t w = work_item(blockIdx.x, n);
  if (w >= n) return;
  const uint32_t slot = w / (uint32_t)a.Hv;
  const int h = (int)(w - slot * (uint32_t)a.Hv), hk = h / (a.Hv / a.Hk);
  const Segment sg(a.q, slot);
  if (sg.len == 0) return;
  const int64_t size = DK * DV, own = ((int64_t)sg.s * a.Hv + h) * size;
  const int64_t tk = (sg.t0 * a.Hk + hk) * DK, tv = (sg.t0 * a.Hv + h) * DV;
  PassTiles<DK, DV, NT, T> tiles{{(const T*)a.Q + tk, a.Hk, sq},
                                 {(const T*)a.K + tk, a.Hk, sk},
                                 {(const T*)a.V + tv, a.Hv, sv}};
  Pass ps{};
  ps.q = sq, ps.k = sk, ps.v = sv;
  ps.ldo = (uint32_t)a.Hv * DV;
  ps.out = (T*)a.O + tv;
  ps.start = a.U ? a.U + ((int64_t)slot * a.Hv + h) * size : a.S0 ? a.S0 + own : nullptr;
  ps.fin = a.Sf && sg.j == sg.n - 1 ? a.Sf + own : nullptr;
  walk<DK, DV, NS, T, kO, false, false>(a, sg, h, ps, tiles, &lds);
}

// ---- the gradients.  A workgroup is two teams of four waves on common tiles (read apart, the
// tiles of the passes came from HBM each time: they run at different places of a segment):
// of a group of two heads, or each two of a larger even one, dQ, dK or dV of both (the first
// team adds up dQ and dK); of one head, or of an odd group's one after the other, dK and dV,
// and dQ by a team of its own.

namespace {

// What dQ (or dK) of value head h takes and gives.
template <int DK, int DV, typename T, Kind P, bool DG>
__device__ __forceinline__ Pass key_pass(const LinArgs& a, const Segment& sg, uint32_t slot, int hk,
                                         int h) {
  constexpr bool rev = P == kDK;
  constexpr int64_t size = DK * DV;
  const int64_t tk = (sg.t0 * a.Hk + hk) * DK;
  const int64_t own = ((int64_t)sg.s * a.Hv + h) * size, at = ((int64_t)slot * a.Hv + h) * size;
  const float* S = a.U ? a.U + at : a.S0 ? a.S0 + own : nullptr;
  Pass ps{};
  ps.ldo = (uint32_t)a.Hk * DK;
  ps.out = (T*)(rev ? a.dK : a.dQ) + tk;
  ps.start = !rev ? S : a.R ? a.R + at : a.dSf ? a.dSf + own : nullptr;
  if (DG) {
    const int64_t tokens = a.q.tokens();
    ps.x = (const T*)(rev ? a.K : a.Q) + tk;
    ps.rows = (rev ? a.rows_k : a.rows_q) + h * tokens + sg.t0;
    ps.against = S;
    ps.anchor = a.anchor + (int64_t)slot * a.Hv + h;
  }
  return ps;
}
template <int DK, int DV, typename T>
__device__ __forceinline__ Pass value_pass(const LinArgs& a, const Segment& sg, uint32_t slot,
                                           int h) {
  constexpr int64_t size = DK * DV;
  const int64_t own = ((int64_t)sg.s * a.Hv + h) * size;
  Pass ps{};
  ps.ldo = (uint32_t)a.Hv * DV;
  ps.out = (T*)a.dV + (sg.t0 * a.Hv + h) * DV;
  ps.start = a.R ? a.R + ((int64_t)slot * a.Hv + h) * size : a.dSf ? a.dSf + own : nullptr;
  ps.fin = a.dS0 && sg.j == 0 ? a.dS0 + own : nullptr;
  return ps;
}

// dQ or dK of a key head with an even group: its value heads two by two
template <int DK, int DV, typename T, Kind P, bool DG>
__device__ __forceinline__ void key_gradient_by_two(const LinArgs& a, const Segment& sg,
                                                    uint32_t slot, int hk, T* s, float* other,
                                                    TeamLds<4, T>* lds) {
  constexpr bool rev = P == kDK, more = rev && DG;
  const int gr = a.Hv / a.Hk, team = __builtin_amdgcn_readfirstlane(threadIdx.x >> 8);
  constexpr int VT = LC * DV, KT = LC * DK;
  const int64_t tk = (sg.t0 * a.Hk + hk) * DK;
  for (int u = 0; u < gr; u += 2) {
    const int h = hk * gr + u;
    const T* q = (const T*)(rev ? a.V : a.dO) + (sg.t0 * a.Hv + h) * DV;
    const T* k = (const T*)(rev ? a.dO : a.V) + (sg.t0 * a.Hv + h) * DV;
    const T *v = (const T*)(rev ? a.Q : a.K) + tk, *x = (const T*)a.K + tk;
    FourAndMore<DV, DK, 512, T, more> tiles{{q, a.Hv, s},
                                            {k, a.Hv, s + VT},
                                            {q + DV, a.Hv, s + 2 * VT},
                                            {k + DV, a.Hv, s + 3 * VT},
                                            {v, a.Hk, s + 4 * VT},
                                            {x, a.Hk, s + 4 * VT + KT}};
    Pass ps = key_pass<DK, DV, T, P, DG>(a, sg, slot, hk, h + team);
    ps.q = s + 2 * team * VT, ps.k = s + (2 * team + 1) * VT, ps.v = s + 4 * VT;
    if (more) ps.x = s + 4 * VT + KT;
    ps.acc = gr > 2 ? (rev ? a.acc_k : a.acc_q) + tk : nullptr;
    ps.first = u == 0, ps.last = u == gr - 2;
    walk<DV, DK, DK / 64, T, P, DG, more>(a, sg, h + team, ps, tiles, lds + team, other);
    lds_only_barrier();
  }
}

}  // namespace

// groups of even size.  (4 x 8192 tokens, 32 heads in pairs: 1.1 to 1.3 ms, 2.5 TB/s, vector units
// busy 45 % and matrix units 30 %.)
template <int DK, int DV, typename T, bool DG>
__global__ __launch_bounds__(512, 2) void k_lin_backward_by_two(const LinArgs a, uint32_t slots) {
  // the second team's results go where the tiles of products lie, which the first has done with
  __shared__ __attribute__((aligned(16))) T s[LC * (4 * DV + (DG ? 2 : 1) * DK)];
  static_assert(4 * DV * sizeof(T) >= DK * sizeof(float) && 2 * DV >= DK, "what else lies there");
  float* other = (float*)s;
  __shared__ __attribute__((aligned(16))) TeamLds<4, T> lds[2];
  const uint32_t nk = slots * (uint32_t)a.Hk, nv = slots * (uint32_t)(a.Hv / 2);
  const uint32_t bk = (2 * nk + 7) & ~7u, bv = (nv + 7) & ~7u;
  if (blockIdx.x >= bk + bv) return copy_state(a, (int)(blockIdx.x - bk - bv), a.dSf, a.dS0);
  const bool keys = blockIdx.x < bk;
  const uint32_t w = keys ? work_item(blockIdx.x, 2 * nk) : work_item(blockIdx.x - bk, nv);
  if (w >= (keys ? 2 * nk : nv)) return;
  const uint32_t heads = (uint32_t)(keys ? a.Hk : a.Hv / 2), v = keys && w >= nk ? w - nk : w;
  const uint32_t slot = v / heads;
  const int i = (int)(v - slot * heads);
  const Segment sg(a.q, slot);
  if (sg.len == 0) return;
  if (keys && w >= nk) {
    key_gradient_by_two<DK, DV, T, kDK, DG>(a, sg, slot, i, s, other, lds);
  } else if (keys) {
    key_gradient_by_two<DK, DV, T, kDQ, DG>(a, sg, slot, i, s, other, lds);
  } else {
    const int team = __builtin_amdgcn_readfirstlane(threadIdx.x >> 8), h = 2 * i;
    const int64_t tk = (sg.t0 * a.Hk + h / (a.Hv / a.Hk)) * DK, tv = (sg.t0 * a.Hv + h) * DV;
    constexpr int KT = LC * DK, VT = LC * DV;
    TwoAndTwo<DK, DV, 512, T> tiles{{(const T*)a.K + tk, a.Hk, s},
                                    {(const T*)a.Q + tk, a.Hk, s + KT},
                                    {(const T*)a.dO + tv, a.Hv, s + 2 * KT},
                                    {(const T*)a.dO + tv + DV, a.Hv, s + 2 * KT + VT}};
    Pass ps = value_pass<DK, DV, T>(a, sg, slot, h + team);
    ps.q = s, ps.k = s + KT, ps.v = s + 2 * KT + team * VT;
    walk<DK, DV, DV / 64, T, kDV, false, false>(a, sg, h + team, ps, tiles, lds + team);
  }
}

// dK and dV of a key head's value heads one after the other.  (8192 tokens of 16 heads: 99 us,
// 2.4 TB/s, vector units busy 41 % and matrix units 27 %.)
template <int DK, int DV, typename T, bool DG>
__global__ __launch_bounds__(512, 2) void k_lin_backward_kv(const LinArgs a, uint32_t slots) {
  constexpr int KT = LC * DK, VT = LC * DV;
  __shared__ __attribute__((aligned(16))) T s[2 * KT + 2 * VT];
  __shared__ __attribute__((aligned(16))) TeamLds<4, T> lds[2];
  const uint32_t n = slots * (uint32_t)a.Hk, blocks = (n + 7) & ~7u;
  if (blockIdx.x >= blocks) return copy_state(a, (int)(blockIdx.x - blocks), a.dSf, a.dS0);
  const uint32_t w = work_item(blockIdx.x, n);
  if (w >= n) return;
  const uint32_t slot = w / (uint32_t)a.Hk;
  const int hk = (int)(w - slot * (uint32_t)a.Hk), gr = a.Hv / a.Hk;
  const int team = __builtin_amdgcn_readfirstlane(threadIdx.x >> 8);
  const Segment sg(a.q, slot);
  if (sg.len == 0) return;
  T *sQ = s, *sK = s + KT, *sV = s + 2 * KT, *sO = s + 2 * KT + VT;
  for (int u = 0; u < gr; ++u) {
    const int h = hk * gr + u;
    const int64_t tk = (sg.t0 * a.Hk + hk) * DK, tv = (sg.t0 * a.Hv + h) * DV;
    TwoAndTwo<DK, DV, 512, T> tiles{{(const T*)a.Q + tk, a.Hk, sQ},
                                    {(const T*)a.K + tk, a.Hk, sK},
                                    {(const T*)a.V + tv, a.Hv, sV},
                                    {(const T*)a.dO + tv, a.Hv, sO}};
    if (team == 0) {
      Pass ps = key_pass<DK, DV, T, kDK, DG>(a, sg, slot, hk, h);
      ps.q = sV, ps.k = sO, ps.v = sQ, ps.x = sK;
      ps.acc = gr > 1 ? a.acc_k + tk : nullptr;
      ps.first = u == 0, ps.last = u == gr - 1;
      walk<DV, DK, DK / 64, T, kDK, DG, true>(a, sg, h, ps, tiles, lds);
    } else {
      Pass ps = value_pass<DK, DV, T>(a, sg, slot, h);
      ps.q = sK, ps.k = sQ, ps.v = sO;
      walk<DK, DV, DV / 64, T, kDV, false, false>(a, sg, h, ps, tiles, lds + 1);
      if (DG) lds_only_barrier();  // (the other team's, before its last rows)
    }
    lds_only_barrier();
  }
}

// one of the gradients by a team of its own
template <int DK, int DV, typename T, Kind P, bool DG>
__global__ __launch_bounds__(256, kGroups<T>) void k_lin_backward(const LinArgs a, uint32_t n) {
  constexpr bool keys = kFlipped<P>;
  constexpr int D0 = keys ? DV : DK, D1 = keys ? DK : DV;  // of the products, of the result
  __shared__ __attribute__((aligned(16))) T sq[LC * D0], sk[LC * D0], sv[LC * D1];
  __shared__ __attribute__((aligned(16))) TeamLds<4, T> lds;
  const uint32_t blocks = (n + 7) & ~7u;
  if (blockIdx.x >= blocks) return copy_state(a, (int)(blockIdx.x - blocks), a.dSf, a.dS0);
  const uint32_t w = work_item(blockIdx.x, n);
  if (w >= n) return;
  const uint32_t heads = (uint32_t)(keys ? a.Hk : a.Hv), slot = w / heads;
  const int i = (int)(w - slot * heads), gr = a.Hv / a.Hk, hk = keys ? i : i / gr;
  const Segment sg(a.q, slot);
  if (sg.len == 0) return;
  const T *Q = (const T*)a.Q, *K = (const T*)a.K, *V = (const T*)a.V, *dO = (const T*)a.dO;
  for (int u = 0; u < (keys ? gr : 1); ++u) {
    const int h = keys ? hk * gr + u : i;
    const int64_t tk = (sg.t0 * a.Hk + hk) * DK, tv = (sg.t0 * a.Hv + h) * DV;
    const int Hq = keys ? a.Hv : a.Hk, Ho = keys ? a.Hk : a.Hv;
    PassTiles<D0, D1, 256, T> tiles{
        {P == kDQ ? dO + tv : P == kDK ? V + tv : K + tk, Hq, sq},
        {P == kDQ ? V + tv : P == kDK ? dO + tv : Q + tk, Hq, sk},
        {P == kDQ ? K + tk : P == kDK ? Q + tk : dO + tv, Ho, sv}};
    Pass ps;
    if constexpr (keys) {
      ps = key_pass<DK, DV, T, P, DG>(a, sg, slot, hk, h);
      ps.acc = gr > 1 ? (P == kDK ? a.acc_k : a.acc_q) + tk : nullptr;
      ps.first = u == 0, ps.last = u == gr - 1;
    } else {
      ps = value_pass<DK, DV, T>(a, sg, slot, h);
    }
    ps.q = sq, ps.k = sk, ps.v = sv;
    walk<D0, D1, D1 / 64, T, P, DG, false>(a, sg, h, ps, tiles, &lds);
    lds_only_barrier();
  }
}

// ---- the gradient of g from the rows' sums; a wave takes a chunk.  (18 us for 4 x 8192 tokens of
// 32 heads, one value a head and token written in each line of 128 bytes; 6 and 4 for the sums of
// a head's decay over 8192 tokens of 16.)
__global__ __launch_bounds__(256) void k_lin_decay(const LinArgs a) {
  __shared__ float sq[kMostChunks], sk[kMostChunks], wave[4];
  const uint32_t slot = blockIdx.x / (uint32_t)a.Hv;
  const int h = (int)(blockIdx.x - slot * (uint32_t)a.Hv);
  const int w = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), l = lane_id();
  const Segment sg(a.q, slot);
  const int64_t at = (int64_t)slot * a.Hv + h;
  const int64_t tokens = a.q.tokens();
  const float* rq = a.rows_q + h * tokens + sg.t0;
  const float* rk = a.rows_k + h * tokens + sg.t0;
  const int nc = (sg.len + LC - 1) / LC;
  for (int c = w; c < nc; c += 4) {
    const int t = c * LC + l;
    const float q = sum_lanes<64>(t < sg.len ? rq[t] : 0.f);
    const float k = sum_lanes<64>(t < sg.len ? rk[t] : 0.f);
    if (l == 0) sq[c] = q, sk[c] = k;
  }
  __syncthreads();
  float all = 0.f;
  for (int c = w; c < nc; c += 4) {
    float x = a.anchor[at];  // X of the first chunk, and from there X of this one
    for (int i = 1; i <= c; ++i) x += sk[i - 1] - sq[i];
    const int t = c * LC + l;
    const float q = t < sg.len ? rq[t] : 0.f, k = t < sg.len ? rk[t] : 0.f;
    const double pq = prefix64((double)q), pk = prefix64((double)k);
    x += (float)((lane63(pq) - (pq - q)) + (pk - k));
    if (t < sg.len) {
      if (a.per_token) a.dg[(sg.t0 + t) * a.Hv + h] = x;
      all += x;
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

// Tokens a segment.  Short ones fill the chip, long ones save launches and states (each is
// written, carried over the segments and read: 4 times 64 KB, 9 in the backward pass): the one
// of least time by what the launches took, in us, for heads of 128 by 128 in bf16.  A step
// of a walk, of 64 tokens, takes 4.6 with one workgroup a CU and 3.6 to 3.8 each with two, forming
// a segment's state 1.2 and 0.9; 11 to 12 a step of two teams, one workgroup a CU; with fp32
// inputs 3.8 times as long.  (Forward, 16 heads of 8192 tokens: 128 us in segments of 64, 101 of
// 128, 79 of 256, 79 to 82 of 512, 98 of 768, 175 of 1536; 4 of 1000: 23 of 64, 26 of 128, 37 of
// 256, 83 in one, in fp32 34, 49, 85 and 221.  Gradients, 16 heads of 8192: 443 of 64, 226 of 256,
// 210 of 512, 318 of 1024; 32 of 2 x 8192 with 16 key heads: 866 of 256, 738 of 512, 670 of 1024.
// Packed, 16384 tokens in 31 sequences, 16 heads: forward 325, 228, 181, 196, 200 of 64, 128, 256,
// 512, 1024; gradients, 8 key heads: 982, 648, 530, 503, 592.  Over nine packed mixes the segments
// chosen take 4 % more than the best ones, 2 % for the gradients.)
int lin_segment(int nseq, int T, int Hk, int Hv, int dk, int dv, bool packed, bool backward,
                bool fp32) {
  const double tokens = packed ? (double)T : (double)nseq * T, gr = Hk ? (double)Hv / Hk : 1;
  const double size = (0.25 + 0.75 * dk * dv / 16384) * (fp32 ? 3.8 : 1);
  const int most = backward ? LC * kMostChunks : 4096;
  const int64_t whole = ((int64_t)T + LC - 1) / LC * LC;
  int best = LC;
  double least = 1e300;
  for (int k = 1;; k += k < 8 ? 1 : k < 16 ? 2 : k < 32 ? 4 : 8) {
    int64_t seg = std::min<int64_t>((int64_t)k * LC, most);
    const bool one = seg >= whole;
    if (one) seg = std::max<int64_t>(whole, LC);
    const double steps = (double)seg / LC;
    const double slots = packed ? tokens / seg + 0.5 * nseq : std::ceil((double)T / seg) * nseq;
    // steps of `work` walkers on 256 CUs, `places` on each (equal ones in whole rounds; of unlike
    // ones the last begins late: half a round's more).  Packed sequences' segments are of all
    // lengths, some slots empty: the steps there are, and what begins late.
    auto time = [&](double work, double alone, double more, double whole_rounds, int places) {
      double n = work / 256;
      if (packed) {
        n *= (tokens / LC + 0.5 * nseq + 0.8 * slots) / (slots * steps);
        n += 0.5 * (std::ceil(n / places) * places - n);
      } else {
        n += whole_rounds * (std::ceil(n) - n);
      }
      const double t = steps * (fp32 ? alone * std::max(1., n) : std::max(alone, more * n));
      return packed ? t + (backward ? 0.25 : 2) * steps * alone : t;
    };
    const double states = slots * Hv;
    double walk, add = time(backward ? 2 * states : states, 1.2, 0.9, 1, 2);
    if (!backward)
      walk = time(states, 4.6, 3.6, 1, 2);
    else if (!fp32 && Hk && Hv / Hk % 2 == 0)
      walk = time(1.5 * states, 5.5 * gr, 11, 0.5, 1);  // (a group's pairs one after the other)
    else
      walk = gr * (time(slots * Hk, 12, 12, 0, 1) + time(slots * Hk, 6, 4.5, 1, 2));
    double cost = size * (walk + (one ? 0 : add)) + (one ? 4 : 12);
    if (!one) cost += states * (backward ? 0.131 : 0.058) * dk * dv / 16384;
    if (cost < least) least = cost, best = (int)seg;
    if (one || k * LC >= most) break;
  }
  return best;
}

int64_t lin_workspace(LinArgs& a, bool backward, float* ws) {
  const int64_t slots = a.q.slots(), size = (int64_t)a.dk * a.dv;
  const int64_t tokens = a.q.tokens();
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
    constexpr int NS = kStateBlocks;
    if (dtype == 0)
      hipLaunchKernelGGL((k_lin_state<DK, DV, NS, float>), dim3(grid), dim3(4 * DV / NS), 0, st, a,
                         n, both);
    else
      hipLaunchKernelGGL((k_lin_state<DK, DV, NS, __bf16>), dim3(grid), dim3(4 * DV / NS), 0, st,
                         a, n, both);
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
      hipLaunchKernelGGL((k_lin_forward<DK, DV, float>), dim3(grid), dim3(256), 0, st, a, n);
    else
      hipLaunchKernelGGL((k_lin_forward<DK, DV, __bf16>), dim3(grid), dim3(256), 0, st,
                         a, n);
    return hipGetLastError();
  }))
  return hipErrorNotSupported;
}

// the gradients' launches
template <int DK, int DV, bool DG>
static hipError_t launch_passes(const LinArgs& a, uint32_t slots, int dtype, hipStream_t st) {
  const uint32_t nk = slots * a.Hk, nv = slots * a.Hv;
  const uint32_t copies = a.dS0 && (a.q.cu || a.q.T == 0) ? a.q.nseq : 0;
  auto grid = [](uint32_t n, uint32_t more) { return dim3(((n + 7) & ~7u) + more); };
  if (slots == 0) {
    if (!copies) return hipSuccess;
    hipLaunchKernelGGL((k_lin_backward<DK, DV, float, kDV, false>), grid(0, copies),
                       dim3(256), 0, st, a, 0);
  } else if (dtype == 0) {
    hipLaunchKernelGGL((k_lin_backward<DK, DV, float, kDQ, DG>), grid(nk, 0), dim3(256), 0,
                       st, a, nk);
    if (hipError_t e = hipGetLastError()) return e;
    hipLaunchKernelGGL((k_lin_backward<DK, DV, float, kDK, DG>), grid(nk, 0), dim3(256), 0,
                       st, a, nk);
    if (hipError_t e = hipGetLastError()) return e;
    hipLaunchKernelGGL((k_lin_backward<DK, DV, float, kDV, false>), grid(nv, copies),
                       dim3(256), 0, st, a, nv);
  } else if (a.Hv / a.Hk % 2 == 0) {
    const uint32_t blocks = ((2 * nk + 7) & ~7u) + ((nv / 2 + 7) & ~7u);
    hipLaunchKernelGGL((k_lin_backward_by_two<DK, DV, __bf16, DG>),
                       dim3(blocks + copies), dim3(512), 0, st, a, slots);
  } else {
    hipLaunchKernelGGL((k_lin_backward<DK, DV, __bf16, kDQ, DG>), grid(nk, 0),
                       dim3(256), 0, st, a, nk);
    if (hipError_t e = hipGetLastError()) return e;
    hipLaunchKernelGGL((k_lin_backward_kv<DK, DV, __bf16, DG>), grid(nk, copies),
                       dim3(512), 0, st, a, slots);
  }
  return hipGetLastError();
}

hipError_t launch_linear_backward(const LinArgs& a, int dtype, hipStream_t st) {
  if (a.U)
    if (hipError_t e = launch_states(a, dtype, true, st)) return e;
  const uint32_t slots = a.q.T > 0 ? (uint32_t)a.q.slots() : 0;
  hipError_t e = hipErrorNotSupported;
  GDN_DK_SWITCH(a.dk, GDN_DV_SWITCH(a.dv, {
    e = a.want_dg ? launch_passes<DK, DV, true>(a, slots, dtype, st)
                  : launch_passes<DK, DV, false>(a, slots, dtype, st);
    break;
  }) break;)
  if (e != hipSuccess) return e;
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
