// walk.hip -- the two walks of the backward pass along the chunks of a (sequence,
// value head): the states entering the chunks, first chunk to last, and the
// gradients of the states leaving them, last to first (backward.hip states the
// products).  Value columns do not meet, so a walk is cut into slices of 16.
//
// Bound: a chunk's step is a chain of three dependent products, K S, T Z and K^T Y
// (K dS, T^T dY and K^T dX), a hundred kilobytes of operands apart from the next,
// in the one wave or the team of four that owns the slice's state; past as many
// slices as SIMDs, HBM (the states themselves: 64 KB a chunk): 4 x 8192 tokens of 32 heads of 128 by
// 128 in bf16 take 1.29 ms and move 6 GB, 4.7 TB/s.
#include "backward.hpp"

#include <algorithm>

namespace gdn {

namespace {

// ---- bf16 inputs
// One wave a slice holds the state's [dk, 16] part and forms everything of a chunk's
// step by itself, in fragments that chain from one product to the next in
// registers, without an exchange.  Two more waves of the workgroup copy the next
// chunks' K (Q), T, V (dO) and gates into LDS by DMA, so that neither the copies nor
// their waits lie in the chain.
//   NSL: slices a workgroup; REV: the walk from the last chunk; R: chunks in the LDS
//   ring (of Q two)
template <int DK, int DV, int NSL, bool REV, int R>
struct Flow {
  typedef __bf16 T;
  typedef bf16x4 F;
  static constexpr int NS = DV / 16, NG = NS / NSL;  // slices, workgroups a head
  static constexpr int NQ = DK / 32, NB = 2 * NQ;  // pairs and blocks of state rows
  static constexpr int CW = NSL, LW = 2, B = 64 * (CW + LW);
  static constexpr int KD = DK, VD = DV, RING = R, TB = 16 * 20;
  static constexpr bool BACK = REV;
  static_assert(!REV || R == 2, "");
  // LDS of a chunk, in values of T
  static constexpr int oK = 0, oT = oK + BC * DK, oV = oT + 18 * 512, oR = oV + BC * 16 * NSL;
  static constexpr int BUF = oR + 512;
  struct Lds {
    T sm[R][BUF], sq2[2][REV ? BC * DK : 8];
    float tr[CW][2 * TB];
  };
  // rows of K and Q in 16-byte pieces, piece p of row r at p ^ (r & SW): the 16 rows that
  // a wave reads one piece of lie in different banks
  static constexpr int CPR = DK / 8, SW = CPR - 1, RPI = 64 / CPR;
  static constexpr int KC = BC / RPI, VPR = 2 * NSL, VC = BC * VPR / 64;  // copies of 1 KB
  // copies a loader wave and step: of Q, and of the rest (one more of the first wave)
  static constexpr int QN = REV ? KC / 2 : 0, KN = KC / 2 + 9 + VC / 2;
  static_assert(CPR <= 16 && QN + KN + 1 < 64, "vmcnt counts to 63");
  static __device__ __forceinline__ int at(int r, int col) {
    return r * DK + (((col >> 3) ^ (r & SW)) << 3) + (col & 7);
  }
  static __device__ __forceinline__ Pair<F> row_pair(const T* s, int r0, int c0, Lane ln) {
    const int r = r0 + ln.c(), k = c0 + 4 * ln.g();
    return join(*(const bf16x4*)(s + at(r, k)), *(const bf16x4*)(s + at(r, k + 16)));
  }
  static __device__ __forceinline__ Pair<F> col_pair(const T* s, int r0, int c0, Lane ln) {
    const int r = r0 + 4 * ln.g() + (ln.c() >> 2), k = c0 + 4 * (ln.c() & 3);
    return join(read_transposed(s + at(r, k)), read_transposed(s + at(r + 16, k)));
  }
  // the pair (I, p) of T^T: the blocks (2p, I) and (2p + 1, I) of T's fragments,
  // transposed.  Lane l of a slot holds T's row l % 16, columns 4 (l / 16) ...
  static __device__ __forceinline__ Terms<F> t_rows(const T* s, int I, int p, Lane ln) {
    const T* at = s + 8 * (16 * (ln.c() & 3) + 4 * ln.g() + (ln.c() >> 2)) + 4 * (I & 1);
    Terms<F> r;
#pragma unroll
    for (int i = 0; i < 3; ++i)
      r.t[i] = join(read_transposed(slot_at(at, t_slot(2 * p, I >> 1), i, 3)),
                    read_transposed(slot_at(at, t_slot(2 * p + 1, I >> 1), i, 3)));
    return r;
  }
  // column-form block of rows r0 .. and 16 columns c0 .. of the slices' rows of V (dO)
  static __device__ __forceinline__ f32x4 val_block(const T* s, int r0, int c0, Lane ln) {
    const int r = r0 + 4 * ln.g() + (ln.c() >> 2);
    return __builtin_convertvector(
        read_transposed(s + r * 16 * NSL + c0 + 4 * (ln.c() & 3)), f32x4);
  }
  // one wave's copy of 16 bytes a lane into 1 KB of LDS
  static __device__ __forceinline__ void copy(T* to, const void* from) {
    __builtin_amdgcn_global_load_lds((glb_void*)from, (lds_void*)to, 16, 0, 0);
  }
};

}  // namespace

template <typename W>
__device__ __forceinline__ void lone_waves(const BwdArgs& a, typename W::Lds& lds, unsigned bx) {
  constexpr int DK = W::KD, DV = W::VD, NSL = W::CW, R = W::RING;
  constexpr bool REV = W::BACK;
  typedef __bf16 T;
  typedef bf16x4 F;
  constexpr int NQ = W::NQ, NB = W::NB, TB = W::TB;
  auto& sm = lds.sm;
  auto& sq2 = lds.sq2;
  auto& tr = lds.tr;
  // Workgroups are dealt to the 8 XCDs in turn; all those of a head go to one, whose
  // L2 then reads the head's chunks once.
  const unsigned xr = bx >> 3;
  const int64_t sh = (int64_t)(xr / W::NG) * 8 + (bx & 7);
  if (sh >= (int64_t)a.nseq * a.Hv) return;  // the whole workgroup, before any barrier
  const int n0 = (int)(xr % W::NG) * 16 * NSL, s = (int)((uint32_t)sh / (uint32_t)a.Hv);
  const int h = (int)((uint32_t)sh - (uint32_t)s * (uint32_t)a.Hv), hk = h / a.gr;
  const Seq sq(a, s);
  const int wv = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), nc = sq.chunks();
  const Lane ln = lane_here();
  const int l = ln.id, g = ln.g(), c = ln.c();
  const int64_t vld = (int64_t)a.Hv * DV;
  auto tile = [&](int ck) { return a.ws + ((sq.base + ck) * a.Hv + h) * ws_tile(DK, DV); };
  auto rows = [&](int ck) { return min(BC, sq.len - ck * BC); };
  auto chunk = [&](int i) { return REV ? nc - 1 - i : i; };  // of step i

  if (wv >= W::CW) {
    if (wv >= W::CW + W::LW) return;  // (a workgroup of both kinds has two waves more)
    // ---- loader.  Step i's operands are read between the barrier that ends step
    // i - 1 and the one that ends step i.  Rows past a chunk's last token repeat it: their beta is 0, which takes them
    // out of Z and dX, and dO's are masked where they are used.  Steps past the
    // last load its operands again, into buffers that no step reads.
    const int lw = wv - W::CW;
    const uint32_t kld = (uint32_t)a.Hk * DK * 2, vb = (uint32_t)vld * 2;
    const int lr = l / W::CPR, lp = l % W::CPR;
    auto load_rows = [&](const void* p, int ck, T* to) __attribute__((always_inline)) {
      const char* from = (const char*)((const T*)p + ((sq.t0 + (int64_t)ck * BC) * a.Hk + hk) * DK);
      const int m = rows(ck);
#pragma unroll
      for (int i = 0; i < W::KC / 2; ++i) {
        const int r = (2 * i + lw) * W::RPI + lr;
        W::copy(to + (2 * i + lw) * 512, from + (min(r, m - 1) * kld + ((lp ^ (r & W::SW)) << 4)));
      }
    };
    auto load = [&](int i) __attribute__((always_inline)) {
      const int ck = chunk(min(i, nc - 1)), m = rows(ck);
      T* to = sm[i % R];
      const float* ws = tile(ck);
      load_rows(a.K, ck, to + W::oK);
      const float* t = ws + ws_T() + 4 * l;
#pragma unroll
      for (int k = 0; k < 9; ++k)
        W::copy(to + W::oT + (2 * k + lw) * 512, t + (2 * k + lw) * 256);
      const char* V = (const char*)((const T*)(REV ? a.dO : a.V) +
                                    ((sq.t0 + (int64_t)ck * BC) * a.Hv + h) * DV + n0);
#pragma unroll
      for (int k = 0; k < W::VC / 2; ++k) {
        const int r = (2 * k + lw) * (64 / W::VPR) + l / W::VPR;
        W::copy(to + W::oV + (2 * k + lw) * 512, V + (min(r, m - 1) * vb + l % W::VPR * 16));
      }
      if (lw == 0) W::copy(to + W::oR, ws + ws_rows() + 4 * l);
    };
    auto load_q = [&](int i) __attribute__((always_inline)) {
      if (REV) load_rows(a.Q, chunk(min(i, nc - 1)), sq2[i & 1]);
    };
    if (nc > 0) {
      load_q(0);
      load(0);
      if (R > 2) load(1);
      wait_vmem();
      copier_barrier();
      for (int i = 0; i < nc; ++i) {
        load_q(i + 1);
        load(i + R - 1);
        if (R > 2) {  // all but this step's
          constexpr int n0 = W::QN + W::KN + 1, n1 = n0 - 1;
          if (lw == 0)
            __builtin_amdgcn_s_waitcnt(0x0F70 | (n0 & 15) | ((n0 >> 4) << 14));
          else
            __builtin_amdgcn_s_waitcnt(0x0F70 | (n1 & 15) | ((n1 >> 4) << 14));
        }
        if (R == 2) wait_vmem();
        copier_barrier();
      }
      wait_vmem();  // before the LDS is another workgroup's
    }
    return;
  }

  // ---- the wave of slice wv
  const int sl = wv, J = n0 / 16 + sl;
  const float* init = REV ? a.dSf : a.S0;
  f32x4 st[NB];
#pragma unroll
  for (int b = 0; b < NB; ++b)
    st[b] = init ? col_block(init + sh * DK * DV + 16 * J, DV, 16 * b, DK) : zero4();
  f32x4 r[4];  // R, asked for a chunk ahead
  auto fetch_r = [&](int ck) __attribute__((always_inline)) {
    const float* p = tile(ck) + ws_R() + 4 * l;
#pragma unroll
    for (int I = 0; I < 4; ++I) r[I] = at4(p + blk_at(I, J, W::NS));
  };
  if (REV && nc > 0) fetch_r(chunk(0));
  if (nc > 0) lds_only_barrier();
  for (int i = 0; i < nc; ++i) {
    const int ck = chunk(i);
    const T* buf = sm[i % R];
    const T *sK = buf + W::oK, *sQ = sq2[i & 1], *sT = buf + W::oT, *sV = buf + W::oV;
    const float* rv = (const float*)(buf + W::oR) + 4 * g;  // beta, e^gamma, e^{gl - gamma}
    float* ws = tile(ck);
    // K S (K dS)
    f32x4 x[4];
#pragma unroll
    for (int I = 0; I < 4; ++I) x[I] = zero4();
#pragma unroll
    for (int q = 0; q < NQ; ++q) {
      Pair<F> kr[4];
#pragma unroll
      for (int I = 0; I < 4; ++I) kr[I] = W::row_pair(sK, 16 * I, 32 * q, ln);
      mma_in<false, 4>(kr, split<F>(st[2 * q], st[2 * q + 1]), x);
    }
    // the state, for the per-chunk launch: row-form blocks by way of LDS
    float* out = ws + (REV ? ws_dS(DK, DV) : ws_S(DV)) + 4 * l;
#pragma unroll
    for (int q = 0; q < NQ; ++q) {
      float* t = tr[wv];
#pragma unroll
      for (int hf = 0; hf < 2; ++hf)
#pragma unroll
        for (int v = 0; v < 4; ++v) t[TB * hf + (4 * g + v) * 20 + c] = st[2 * q + hf][v];
      lds_sync<true>();
#pragma unroll
      for (int hf = 0; hf < 2; ++hf)
        *(f32x4*)(out + blk_at(2 * q + hf, J, W::NS)) = at4(t + TB * hf + c * 20 + 4 * g);
      lds_sync<true>();
    }
    // Z (dY), then Y (dZ)
    Terms<F> y[2];
    {
      f32x4 z[4];
#pragma unroll
      for (int I = 0; I < 4; ++I) {
        if constexpr (REV) {
          z[I] = r[I] + at4(rv + 2 * BC + 16 * I) * x[I];
        } else {
          const f32x4 xx = W::val_block(sV, 16 * I, 16 * sl, ln) - at4(rv + BC + 16 * I) * x[I];
          *(f32x4*)(ws + ws_X(DV) + blk_at(I, J, W::NS) + 4 * l) = xx;
          z[I] = at4(rv + 16 * I) * xx;
        }
      }
      if constexpr (REV)
        if (i + 1 < nc) fetch_r(chunk(i + 1));
      const Terms<F> zt[2] = {split<F>(z[0], z[1]), split<F>(z[2], z[3])};
      // the six products T (I, p) Z_p, the terms of each kind side by side
      f32x4 u[4], ul[4];
#pragma unroll
      for (int I = 0; I < 4; ++I) u[I] = ul[I] = zero4();
#pragma unroll
      for (int p = 0; p < 2; ++p) {
        Terms<F> ts[4];
#pragma unroll
        for (int k = 0; k < 6; ++k) {
          constexpr int tx[6] = {0, 1, 2, 1, 0, 0}, ty[6] = {2, 1, 0, 0, 1, 0};
#pragma unroll
          for (int I = 0; I < 4; ++I) {
            if (REV ? p < I / 2 : p > I / 2) continue;
            if (k == 0) ts[I] = REV ? W::t_rows(sT, I, p, ln) : load_terms<F>(sT, t_slot(I, p), l);
            f32x4& acc = k & 1 ? u[I] : ul[I];
            acc = Pair<F>::template mma<false>(ts[I].t[tx[k]], zt[p].t[ty[k]], acc);
          }
        }
      }
#pragma unroll
      for (int I = 0; I < 4; ++I) {
        u[I] += ul[I];
        if constexpr (REV) {
          *(f32x4*)(ws + ws_R() + blk_at(I, J, W::NS) + 4 * l) = u[I];
          u[I] = at4(rv + 16 * I) * u[I];  // dX
          const int m = rows(ck), r0 = 16 * I + 4 * g;
          T* dV = (T*)a.dV + ((sq.t0 + (int64_t)ck * BC + r0) * a.Hv + h) * DV + 16 * J + c;
#pragma unroll
          for (int v = 0; v < 4; ++v)
            if (r0 + v < m) dV[v * vld] = (T)u[I][v];
          z[I] = -at4(rv + BC + 16 * I) * u[I];
        } else {
          z[I] = at4(rv + 2 * BC + 16 * I) * u[I];
        }
      }
      y[0] = split<F>(z[0], z[1]);
      y[1] = split<F>(z[2], z[3]);
    }
    // the state that the next step starts from
    const float el = rv[BC + BC - 1 - 4 * g];
    if constexpr (REV) {
      const int m = rows(ck);
      f32x4 o[4];
#pragma unroll
      for (int I = 0; I < 4; ++I) {
        o[I] = W::val_block(sV, 16 * I, 16 * sl, ln) * (at4(rv + BC + 16 * I) * a.scale);
        if (m < 16 * I + 16)
#pragma unroll
          for (int v = 0; v < 4; ++v) o[I][v] = 16 * I + 4 * g + v < m ? o[I][v] : 0.f;
      }
      const Terms<F> ot[2] = {split<F>(o[0], o[1]), split<F>(o[2], o[3])};
#pragma unroll
      for (int q = 0; q < NQ; ++q) {
        f32x4 u[2] = {zero4(), zero4()}, w[2] = {zero4(), zero4()};
        Pair<F> qc[4], kc[4];  // [2 token pair + block]
#pragma unroll
        for (int k = 0; k < 4; ++k) {
          qc[k] = W::col_pair(sQ, 32 * (k >> 1), 32 * q + 16 * (k & 1), ln);
          kc[k] = W::col_pair(sK, 32 * (k >> 1), 32 * q + 16 * (k & 1), ln);
        }
#pragma unroll
        for (int p = 0; p < 2; ++p)
#pragma unroll
          for (int t = 2; t >= 0; --t)
#pragma unroll
            for (int hf = 0; hf < 2; ++hf) {
              u[hf] = Pair<F>::template mma<false>(qc[2 * p + hf], ot[p].t[t], u[hf]);
              w[hf] = Pair<F>::template mma<false>(kc[2 * p + hf], y[p].t[t], w[hf]);
            }
#pragma unroll
        for (int hf = 0; hf < 2; ++hf) st[2 * q + hf] = st[2 * q + hf] * el + (u[hf] + w[hf]);
      }
    } else {
      f32x4 u[NB];
#pragma unroll
      for (int b = 0; b < NB; ++b) u[b] = zero4();
#pragma unroll
      for (int q = 0; q < NQ; ++q) {
        Pair<F> kc[4];  // [2 token pair + block]
#pragma unroll
        for (int k = 0; k < 4; ++k)
          kc[k] = W::col_pair(sK, 32 * (k >> 1), 32 * q + 16 * (k & 1), ln);
#pragma unroll
        for (int p = 0; p < 2; ++p)
#pragma unroll
          for (int t = 2; t >= 0; --t)
#pragma unroll
            for (int hf = 0; hf < 2; ++hf)
              u[2 * q + hf] = Pair<F>::template mma<false>(kc[2 * p + hf], y[p].t[t],
                                                           u[2 * q + hf]);
      }
#pragma unroll
      for (int b = 0; b < NB; ++b) st[b] = st[b] * el + u[b];
    }
    lds_only_barrier();
  }
  if (REV && a.dS0)
#pragma unroll
    for (int b = 0; b < NB; ++b)
#pragma unroll
      for (int v = 0; v < 4; ++v)
        a.dS0[sh * DK * DV + (int64_t)(16 * b + 4 * g + v) * DV + 16 * J + c] =
            st[b][v];
}

// The same walk for few slices, where the step's latency is all: four waves share
// each product of one slice, as with fp32 inputs below (three exchanges a chunk), and
// two more copy the operands.  The loads were in the compute waves' way: their
// counter runs in order with the stores', and waiting for the next chunk's
// operands waited for the last one's states to be written.
// Step i's K is asked for in step i - 2 (after its buffer's rows are in registers),
// the rest in step i - 1.  Four loaders: a copy takes one 60 ns to issue, and the
// barriers wait for it.
template <int DK, int DV, bool REV>
struct Team : Flow<DK, DV, 1, REV, 2> {
  typedef Flow<DK, DV, 1, REV, 2> W;
  static constexpr int LW = 4, B = 64 * (4 + LW), NQ = DK / 32;
  // copies a loader: of K or Q, and of T, V and the gates
  static constexpr int KN = W::KC / LW, QN = REV ? KN : 0, TN = (18 + LW - 1) / LW + 2;
  static constexpr int oT = 0, oV = 18 * 512, oR = oV + BC * 16, oQ = oR + 512;
  static constexpr int BUF = oQ + (REV ? BC * DK : 0);
  struct Lds {
    typename W::T sk[2][BC * DK], sm[2][BUF];
    float part[NQ * 4 * 256], tr[NQ][2 * W::TB];
    typename W::T sZ[6 * 512], sY[6 * 512], sO[REV ? 6 * 512 : 8];
  };
  template <int N>
  static __device__ __forceinline__ void wait() {  // for all but the last N copies
    __builtin_amdgcn_s_waitcnt(0x0F70 | (N & 15) | ((N >> 4) << 14));
  }
};

template <typename W>
__device__ __forceinline__ void team(const BwdArgs& a, typename W::Lds& lds, unsigned bx) {
  constexpr int DK = W::KD, DV = W::VD;
  constexpr bool REV = W::BACK;
  typedef __bf16 T;
  typedef bf16x4 F;
  constexpr int NQ = W::NQ, NS = DV / 16, TB = W::TB;
  auto& sk = lds.sk;
  auto& sm = lds.sm;
  auto& tr = lds.tr;
  float* part = lds.part;
  T *sZ = lds.sZ, *sY = lds.sY, *sO = lds.sO;
  const unsigned xr = bx >> 3;  // all slices of a head on one XCD
  const int64_t sh = (int64_t)(xr / NS) * 8 + (bx & 7);
  if (sh >= (int64_t)a.nseq * a.Hv) return;  // the whole workgroup, before any barrier
  const int J = (int)(xr % NS), s = (int)((uint32_t)sh / (uint32_t)a.Hv);
  const int h = (int)((uint32_t)sh - (uint32_t)s * (uint32_t)a.Hv), hk = h / a.gr;
  const Seq sq(a, s);
  const int wv = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), nc = sq.chunks();
  const Lane ln = lane_here();
  const int l = ln.id, g = ln.g(), c = ln.c();
  const int64_t vld = (int64_t)a.Hv * DV;
  auto tile = [&](int ck) { return a.ws + ((sq.base + ck) * a.Hv + h) * ws_tile(DK, DV); };
  auto rows = [&](int ck) { return min(BC, sq.len - ck * BC); };
  auto chunk = [&](int i) { return REV ? nc - 1 - i : i; };  // of step i

  if (wv >= 4) {
    // ---- loader; steps past the last load its operands again, into buffers that no
    // step reads
    const int lw = wv - 4;
    const uint32_t kld = (uint32_t)a.Hk * DK * 2, vb = (uint32_t)vld * 2;
    const int lr = l / W::CPR, lp = l % W::CPR;
    auto load_rows = [&](const void* p, int i, T* to) __attribute__((always_inline)) {
      const int ck = chunk(min(i, nc - 1)), m = rows(ck);
      const char* from = (const char*)((const T*)p + ((sq.t0 + (int64_t)ck * BC) * a.Hk + hk) * DK);
#pragma unroll
      for (int k = 0; k < W::KN; ++k) {
        const int r = (W::LW * k + lw) * W::RPI + lr;
        W::copy(to + (W::LW * k + lw) * 512,
                from + (min(r, m - 1) * kld + ((lp ^ (r & W::SW)) << 4)));
      }
    };
    // (where a count does not divide, the last copy is made more than once)
    auto load = [&](int i) __attribute__((always_inline)) {
      const int ck = chunk(min(i, nc - 1)), m = rows(ck);
      T* to = sm[i & 1];
      const float* ws = tile(ck);
      const float* t = ws + ws_T() + 4 * l;
#pragma unroll
      for (int k = 0; k < W::TN - 2; ++k) {
        const int n = min(W::LW * k + lw, 17);
        W::copy(to + W::oT + n * 512, t + n * 256);
      }
      const char* V = (const char*)((const T*)(REV ? a.dO : a.V) +
                                    ((sq.t0 + (int64_t)ck * BC) * a.Hv + h) * DV + 16 * J);
      const int r = (lw & 1) * 32 + l / 2;
      W::copy(to + W::oV + (lw & 1) * 512, V + (min(r, m - 1) * vb + l % 2 * 16));
      W::copy(to + W::oR, ws + ws_rows() + 4 * l);
    };
    auto load_q = [&](int i) __attribute__((always_inline)) {
      if (REV) load_rows(a.Q, i, sm[i & 1] + W::oQ);
    };
    if (nc > 0) {
      load_rows(a.K, 0, sk[0]);
      load(0);
      load_rows(a.K, 1, sk[1]);
      load_q(0);
      wait_vmem();
      copier_barrier();
      for (int i = 0; i < nc; ++i) {
        W::template wait<W::KN + W::QN>();  // step i's T, V and gates
        copier_barrier();                 // 1
        load(i + 1);
        W::template wait<W::TN>();  // its Q
        copier_barrier();         // 2: K's buffer is free
        load_rows(a.K, i + 2, sk[i & 1]);
        W::template wait<W::QN + W::TN + W::KN>();  // step i + 1's K
        copier_barrier();                         // 3
        load_q(i + 1);
      }
      wait_vmem();  // before the LDS is another workgroup's
    }
    return;
  }

  const bool owner = wv < NQ;
  const float* init = REV ? a.dSf : a.S0;
  f32x4 st[2];
#pragma unroll
  for (int b = 0; b < 2; ++b)
    st[b] = init && owner ? col_block(init + sh * DK * DV + 16 * J, DV, 32 * wv + 16 * b, DK)
                          : zero4();
  // R of row block wv, asked for two chunks ahead
  f32x4 r0 = zero4(), r1 = zero4();
  auto fetch_r = [&](int i) __attribute__((always_inline)) {
    return at4(tile(chunk(min(i, nc - 1))) + ws_R() + blk_at(wv, J, NS) + 4 * l);
  };
  if (nc > 0) {
    if (REV) {
      r0 = fetch_r(0);
      r1 = fetch_r(1);
    }
    lds_only_barrier();
  }
  auto step = [&](int i, f32x4& r) __attribute__((always_inline)) {
    const int ck = chunk(i);
    const T *sK = sk[i & 1], *buf = sm[i & 1];
    const T *sT = buf + W::oT, *sV = buf + W::oV, *sQ = buf + W::oQ;
    const float* rv = (const float*)(buf + W::oR) + 16 * wv + 4 * g;
    float* ws = tile(ck);
    float* out = ws + (REV ? ws_dS(DK, DV) : ws_S(DV)) + 4 * l;
    Pair<F> kc[4];
    if (owner) {
      Pair<F> kr[4];
#pragma unroll
      for (int I = 0; I < 4; ++I) kr[I] = W::row_pair(sK, 16 * I, 32 * wv, ln);
#pragma unroll
      for (int k = 0; k < 4; ++k)
        kc[k] = W::col_pair(sK, 32 * (k >> 1), 32 * wv + 16 * (k & 1), ln);
      f32x4 x[4];
#pragma unroll
      for (int I = 0; I < 4; ++I) x[I] = zero4();
      mma_in<false, 4>(kr, split<F>(st[0], st[1]), x);
#pragma unroll
      for (int I = 0; I < 4; ++I) *(f32x4*)(part + (4 * wv + I) * 256 + 4 * l) = x[I];
    }
    lds_only_barrier();  // 1
    f32x4 x = zero4();
    {
      f32x4 q[NQ];
#pragma unroll
      for (int k = 0; k < NQ; ++k) q[k] = at4(part + (4 * k + wv) * 256 + 4 * l);
      const f32x4 bt = at4(rv), eg = at4(rv + BC), er = at4(rv + 2 * BC);
      f32x4 v = W::val_block(sV, 16 * wv, 0, ln);
#pragma unroll
      for (int k = 0; k < NQ; ++k) x += q[k];
      if constexpr (REV) {
        store_half<F>(sZ, wv >> 1, wv & 1, split_half<F>(r + er * x), l);
        const int m = rows(ck);
        v *= eg * a.scale;
        if (m < 16 * wv + 16)
#pragma unroll
          for (int k = 0; k < 4; ++k) v[k] = 16 * wv + 4 * g + k < m ? v[k] : 0.f;
        store_half<F>(sO, wv >> 1, wv & 1, split_half<F>(v), l);
        r = fetch_r(i + 2);
      } else {
        x = v - eg * x;
        store_half<F>(sZ, wv >> 1, wv & 1, split_half<F>(bt * x), l);
      }
    }
    // T's row block wv, in the meantime
    Terms<F> tt[2];
#pragma unroll
    for (int p = 0; p < 2; ++p)
      if (REV ? p >= wv / 2 : p <= wv / 2)
        tt[p] = REV ? W::t_rows(sT, wv, p, ln) : load_terms<F>(sT, t_slot(wv, p), l);
    lds_only_barrier();  // 2
    f32x4 u = zero4(), ul = zero4(), w[2] = {zero4(), zero4()};
    {
      Terms<F> z[2];
#pragma unroll
      for (int p = 0; p < 2; ++p)
        if (REV ? p >= wv / 2 : p <= wv / 2) z[p] = load_terms<F>(sZ, p, l);
      // what does not wait for Z: the state, as row-form blocks for the per-chunk launch
      if (owner) {
        float* t = tr[wv];
#pragma unroll
        for (int hf = 0; hf < 2; ++hf)
#pragma unroll
          for (int v = 0; v < 4; ++v) t[TB * hf + (4 * g + v) * 20 + c] = st[hf][v];
      }
#pragma unroll
      for (int p = 0; p < 2; ++p)
        if (REV ? p >= wv / 2 : p <= wv / 2) mma_both<false>(tt[p], z[p], u, ul);
      u += ul;
      const f32x4 bt = at4(rv), eg = at4(rv + BC), er = at4(rv + 2 * BC);
      if constexpr (REV) {
        const f32x4 dx = bt * u;
        store_half<F>(sY, wv >> 1, wv & 1, split_half<F>(-eg * dx), l);
        *(f32x4*)(ws + ws_R() + blk_at(wv, J, NS) + 4 * l) = u;
        const int m = rows(ck), at = 16 * wv + 4 * g;
        T* dV = (T*)a.dV + ((sq.t0 + (int64_t)ck * BC + at) * a.Hv + h) * DV + 16 * J + c;
#pragma unroll
        for (int v = 0; v < 4; ++v)
          if (at + v < m) dV[v * vld] = (T)dx[v];
        if (owner) {
          Pair<F> qc[4];
#pragma unroll
          for (int k = 0; k < 4; ++k)
            qc[k] = W::col_pair(sQ, 32 * (k >> 1), 32 * wv + 16 * (k & 1), ln);
#pragma unroll
          for (int p = 0; p < 2; ++p) {
            const Terms<F> o = load_terms<F>(sO, p, l);
#pragma unroll
            for (int t = 2; t >= 0; --t)
#pragma unroll
              for (int hf = 0; hf < 2; ++hf)
                w[hf] = Pair<F>::template mma<false>(qc[2 * p + hf], o.t[t], w[hf]);
          }
        }
      } else {
        store_half<F>(sY, wv >> 1, wv & 1, split_half<F>(er * u), l);
        *(f32x4*)(ws + ws_X(DV) + blk_at(wv, J, NS) + 4 * l) = x;
      }
      if (owner) {
        const float* t = tr[wv];
        lds_sync<true>();
#pragma unroll
        for (int hf = 0; hf < 2; ++hf)
          *(f32x4*)(out + blk_at(2 * wv + hf, J, NS)) = at4(t + TB * hf + c * 20 + 4 * g);
      }
    }
    const float el = ((const float*)(buf + W::oR))[2 * BC - 1];
    lds_only_barrier();  // 3
    if (owner) {
      f32x4 y[2] = {zero4(), zero4()};
#pragma unroll
      for (int p = 0; p < 2; ++p) {
        const Terms<F> o = load_terms<F>(sY, p, l);
#pragma unroll
        for (int t = 2; t >= 0; --t)
#pragma unroll
          for (int hf = 0; hf < 2; ++hf)
            y[hf] = Pair<F>::template mma<false>(kc[2 * p + hf], o.t[t], y[hf]);
      }
#pragma unroll
      for (int hf = 0; hf < 2; ++hf) st[hf] = st[hf] * el + (w[hf] + y[hf]);
    }
  };
  for (int i = 0; i < nc; i += 2) {
    step(i, r0);
    if (i + 1 < nc) step(i + 1, r1);
  }
  if (REV && a.dS0 && owner)
#pragma unroll
    for (int hf = 0; hf < 2; ++hf)
#pragma unroll
      for (int v = 0; v < 4; ++v)
        a.dS0[sh * DK * DV + (int64_t)(32 * wv + 16 * hf + 4 * g + v) * DV + 16 * J + c] = st[hf][v];
}

// ---- fp32 inputs
// The matrix instructions bound the step (16 times the bf16 ones' time), so four
// waves on the four SIMDs share each product of a slice.  Wave w holds the
// state's rows 32w .. 32w + 31 (two blocks, one pair); a product with the state is
// summed over the waves' own rows (no wave needs another's state), the sums, then
// Z (dY) and Y (dX) of row block w go through LDS, three exchanges a chunk.
template <int DK, int DV>
struct Walk {
  typedef float T;
  typedef f32x4 F;
  static constexpr int NQ = DK / 32, NS = DV / 16;
  static constexpr int E = 4, LD = DK + E;  // rows in LDS, 16 bytes apart
  static constexpr int CPR = DK / E, KI = BC * CPR / 256, TB = 16 * 20;
  typedef f32x4 Vec;
  struct Lds {
    float sK[BC * LD], sQ[BC * LD], part[NQ * 4 * 256], sZ[2 * 512], sY[2 * 512], sO[2 * 512];
    float sT[NQ][2 * TB];
  };
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
  // row block w of T: two pairs at most
  struct TRow {
    Terms<F> v[2];
  };
  static __device__ __forceinline__ void fetch_t(TRow& x, const float* p, int n, int l) {
#pragma unroll
    for (int i = 0; i < 2; ++i)
      if (i < n) x.v[i] = load_terms<F>((const T*)(p + TS * i), 0, l);
  }
  // the same of T^T, from T's fragments: the blocks (J, w), J from the pair of w on
  static __device__ __forceinline__ void fetch_tt(TRow& x, const float* p, int w, Lane ln) {
    const float* at = p + 256 * (w & 1) + 4 * (16 * (ln.c() >> 2) + 4 * ln.g()) + (ln.c() & 3);
#pragma unroll
    for (int i = 0; i < 2; ++i)
      if (i < 2 - w / 2) {
        const int J = 2 * (i + w / 2);
        x.v[i].t[0] = join(down4(at + TS * t_slot(J, w >> 1), 4),
                           down4(at + TS * t_slot(J + 1, w >> 1), 4));
      }
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
template <int DK, int DV>
__device__ __forceinline__ void states_f32(const BwdArgs& a, typename Walk<DK, DV>::Lds& lds) {
  typedef Walk<DK, DV> W;
  typedef float T;
  typedef f32x4 F;
  float *sK = lds.sK, *part = lds.part, *sZ = lds.sZ, *sY = lds.sY;
  auto& sT = lds.sT;
  int n0;
  const int64_t sh = W::head_of(n0);
  if (sh >= (int64_t)a.nseq * a.Hv) return;  // the whole workgroup, before any barrier
  const int s = (int)((uint32_t)sh / (uint32_t)a.Hv);
  const int h = (int)((uint32_t)sh - (uint32_t)s * (uint32_t)a.Hv), hk = h / a.gr;
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
template <int DK, int DV>
__device__ __forceinline__ void reverse_f32(const BwdArgs& a, typename Walk<DK, DV>::Lds& lds) {
  typedef Walk<DK, DV> W;
  typedef float T;
  typedef f32x4 F;
  float *sK = lds.sK, *sQ = lds.sQ, *part = lds.part, *sX = lds.sZ, *sY = lds.sY, *sO = lds.sO;
  auto& sT = lds.sT;
  int n0;
  const int64_t sh = W::head_of(n0);
  if (sh >= (int64_t)a.nseq * a.Hv) return;  // the whole workgroup, before any barrier
  const int s = (int)((uint32_t)sh / (uint32_t)a.Hv);
  const int h = (int)((uint32_t)sh - (uint32_t)s * (uint32_t)a.Hv), hk = h / a.gr;
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
    W::fetch_tt(x.t, ws + ws_T(), wv, ln);
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

// ---- both walks in one launch: neither reads what the other writes, and one of them
// leaves half the chip idle where slices are few.  The slower one goes first.  (One
// after the other, 128 chunks of 16 heads of 128 by 128 in bf16 took 213 + 265 us
// where they take 303 now, 16 chunks in fp32 43 + 62 where they take 64.  Past 256
// slices of fp32 it costs some 8%: 2 x 512 slices of 32 chunks 447 for 415 us, since a
// CU takes two workgroups of the walk over the states alone.)
template <int DK, int DV>
__global__ __launch_bounds__(512) void k_bwd_teams(const BwdArgs a) {
  typedef Team<DK, DV, true> R;
  typedef Team<DK, DV, false> S;
  static_assert(R::B == 512 && S::B == 512, "");
  __shared__ union __attribute__((aligned(16))) {
    typename R::Lds r;
    typename S::Lds s;
  } lds;
  if (blockIdx.y == 0)
    team<R>(a, lds.r, blockIdx.x);
  else
    team<S>(a, lds.s, blockIdx.x);
}

template <int DK, int DV>
__global__ __launch_bounds__(384) void k_bwd_lone(const BwdArgs a) {
  typedef Flow<DK, DV, 4, true, 2> R;
  typedef Flow<DK, DV, 4, false, 3> S;
  static_assert(R::B == 384 && S::B == 384, "");
  __shared__ union __attribute__((aligned(16))) {
    typename R::Lds r;
    typename S::Lds s;
  } lds;
  if (blockIdx.y == 0)
    lone_waves<R>(a, lds.r, blockIdx.x);
  else
    lone_waves<S>(a, lds.s, blockIdx.x);
}

// Packed sequences: those of more than `longest` chunks by teams, first, the others by
// lone waves; the workgroups of the other kind end at once.  (One allocation of registers
// for both: at DK = 128 two values of a lone wave lie in scratch while its loop runs, which
// does not use them.)
template <int DK, int DV>
__global__ __launch_bounds__(512) void k_bwd_mixed(const BwdArgs a, int longest) {
  typedef Team<DK, DV, true> TR;
  typedef Team<DK, DV, false> TS;
  typedef Flow<DK, DV, 4, true, 2> LR;
  typedef Flow<DK, DV, 4, false, 3> LS;
  __shared__ union __attribute__((aligned(16))) {
    typename TR::Lds tr;
    typename TS::Lds ts;
    typename LR::Lds lr;
    typename LS::Lds ls;
  } lds;
  const uint32_t heads = (uint32_t)a.nseq * (uint32_t)a.Hv, n = (heads + 7) / 8 * 8;
  constexpr unsigned NT = DV / 16, NL = DV / 64;  // workgroups a head
  unsigned bx = blockIdx.x;
  const bool teams = bx < 2 * n * NT;
  if (!teams) bx -= 2 * n * NT;
  const unsigned per = teams ? NT : NL, dir = n * per;
  const bool rev = bx < dir;
  if (!rev) bx -= dir;
  const uint32_t sh = (bx >> 3) / per * 8 + (bx & 7);
  if (sh >= heads) return;
  if ((Seq(a, (int)(sh / (uint32_t)a.Hv)).chunks() > longest) != teams) return;
  if (teams) {
    if (rev) team<TR>(a, lds.tr, bx);
    else team<TS>(a, lds.ts, bx);
  } else {
    if (rev) lone_waves<LR>(a, lds.lr, bx);
    else lone_waves<LS>(a, lds.ls, bx);
  }
}

template <int DK, int DV>
__global__ __launch_bounds__(256) void k_bwd_walks_f32(const BwdArgs a) {
  __shared__ __attribute__((aligned(16))) typename Walk<DK, DV>::Lds lds;
  if (blockIdx.y == 0)
    reverse_f32<DK, DV>(a, lds);
  else
    states_f32<DK, DV>(a, lds);
}

template <int DK, int DV>
static hipError_t run_walks(const BwdArgs& a, int dtype, hipStream_t st) {
  const int64_t heads = (int64_t)a.nseq * a.Hv, slices = heads * (DV / 16);
  const unsigned n = (unsigned)((heads + 7) / 8 * 8), both = a.L > 0 ? 2 : 1;
  // A CU takes one team (a slice) or one workgroup of four lone waves (four slices).
  // A team's step takes 2.3 us at most, a workgroup's 4 to 6, so teams walk while both
  // directions' are two rounds: us for 32 chunks, DK = DV = 128, teams and lone waves:
  // 128 slices 70 and 139, 256 133 and 148, 320 190 and 165, 512 281 and 187.
  // Packed sequences differ in length, which the host does not know: all of them by lone
  // waves would keep the CUs busy for about 0.0097 us a chunk and slice, and one of c
  // chunks alone takes 6 c us.  Those that take longer than all together go to teams (the
  // factor is the one that measured best).  8192 tokens of 16 heads by teams alone, lone
  // waves alone, and so: 22 sequences 376, 345, 267 us; 31 372, 321, 277; 9 of at most 30
  // chunks 298, 180, 187; 4 292, 299, 340 (so of few long ones the worst of the three); 8
  // heads in 11 sequences 155, 255, 144.  (Measured for DK = DV = 128.)
  const int64_t longest = (int64_t)a.L * a.Hv * (DV / 16) / 30000;
  if (dtype == 0)
    hipLaunchKernelGGL((k_bwd_walks_f32<DK, DV>), dim3(n * (DV / 16), both), dim3(256), 0, st, a);
  else if (a.cu && a.L > 0)
    hipLaunchKernelGGL((k_bwd_mixed<DK, DV>), dim3((unsigned)packed_walk_groups(a.nseq, a.Hv, DV)),
                       dim3(512), 0, st, a, (int)std::min<int64_t>(longest, INT32_MAX));
  else if (slices <= 256)
    hipLaunchKernelGGL((k_bwd_teams<DK, DV>), dim3(n * (DV / 16), both), dim3(512), 0, st, a);
  else
    hipLaunchKernelGGL((k_bwd_lone<DK, DV>), dim3(n * (DV / 64), both), dim3(384), 0, st, a);
  return hipGetLastError();
}

hipError_t launch_walks(const BwdArgs& a, int dk, int dv, int dtype, hipStream_t st) {
  GDN_DK_SWITCH(dk, GDN_DV_SWITCH(dv, { return run_walks<DK, DV>(a, dtype, st); }))
  return hipErrorNotSupported;
}

}  // namespace gdn
