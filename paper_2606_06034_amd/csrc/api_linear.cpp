// api_linear.cpp -- the extern "C" boundary declared in include/gdnlinear.h.
// Validates every argument before anything is enqueued, then dispatches to
// the launchers.  Holds no state.
#include "gdnlinear.h"

#include <stdint.h>

#include <algorithm>

#include "checks.hpp"
#include "group_norm.hpp"
#include "linear.hpp"

using namespace gdn::checks;

namespace {

// the sizes of a call: its segments, and whether its launches and offsets fit
int set_sizes(gdn::LinArgs& a, const int32_t* cu, bool packed, int nseq, int T, int Hk, int Hv,
              int dk, int dv, bool backward, int dtype) {
  if (nseq < 0 || T < 0 || !valid_heads(Hk, Hv) || !valid_d(dk) || !valid_d(dv))
    return GDN_ERR_SHAPE;
  static const int32_t some = 0;  // (sizes alone are asked for: any offsets)
  a.q.cu = packed ? (cu ? cu : &some) : nullptr;
  a.q.nseq = nseq, a.q.T = T;
  if (!fdtype(dtype)) return GDN_ERR_DTYPE;
  a.q.seg = gdn::lin_segment(nseq, T, Hk, Hv, dk, dv, packed, backward, dtype == GDN_F32);
  a.q.nseg = a.q.segments(T);
  a.Hk = Hk, a.Hv = Hv, a.dk = dk, a.dv = dv;
  const int64_t slots = a.q.slots();
  // workgroups of up to 512 work items: one a segment and head, in the backward pass two or
  // less, one a sequence without tokens, and some left over for each of the 8 XCDs
  if (!grid_ok(slots, 512)) return GDN_ERR_SHAPE;
  if (!grid_ok(slots * Hv * (backward ? 2 : 1) + nseq + 16, 512)) return GDN_ERR_SHAPE;
  return GDN_OK;
}

// rows of a chunk lie at 32-bit offsets from its first (the gradients' sums over the heads of a
// group are fp32).  In reversed time a short chunk's rows are placed from the end of a block of
// 16, which begins before the first: `least` rows.
bool rows_fit(int T, int Hk, int Hv, int dk, int dv, int dtype, int least) {
  const int64_t row = std::max((int64_t)Hk * dk, (int64_t)Hv * dv) * esize(dtype);
  return T == 0 || std::max(least, std::min(T, gdn::LC)) * row <= 1ll << 32;
}

}  // namespace

extern "C" {

int gdn_linear_recurrent(const void* Q, const void* K, const void* V, const float* g,
                         int g_per_token, const float* S0, void* O, float* S_final,
                         const int32_t* slots, int n_states, const int32_t* cu_seqlens, int nseq,
                         int T, int Hk, int Hv, int dk, int dv, float scale, int dtype,
                         void* stream) {
  if (nseq < 0 || T < 0 || n_states < 0 || !valid_heads(Hk, Hv)) return GDN_ERR_SHAPE;
  if (!valid_d(dk) || !valid_d(dv)) return GDN_ERR_SHAPE;
  if (!slots && n_states < nseq && (S0 || S_final)) return GDN_ERR_SHAPE;
  const int64_t heads = (int64_t)nseq * Hv;
  if (heads > 0x7fffffffLL || !grid_ok((heads * (dv / gdn::kStepColumns) + 3) / 4, 256))
    return GDN_ERR_SHAPE;
  if (!fdtype(dtype)) return GDN_ERR_DTYPE;
  if ((int64_t)nseq * Hv == 0) return GDN_OK;
  const int64_t tok = cu_seqlens ? (int64_t)T : (int64_t)nseq * T, es = esize(dtype);
  if (tok > 0 && (!Q || !K || !V || !g || !O)) return GDN_ERR_NULL;
  if (tok == 0) Q = K = V = nullptr, g = nullptr, O = nullptr;
  const int64_t sb = (int64_t)(slots ? n_states : nseq) * Hv * dk * dv * 4;
  const Span in[7] = {{Q, tok * Hk * dk * es},
                      {K, tok * Hk * dk * es},
                      {V, tok * Hv * dv * es},
                      {g, (g_per_token ? tok : 1) * Hv * 4},
                      {S0, sb},
                      {slots, 4ll * nseq},
                      {cu_seqlens, 4ll * (nseq + 1)}};
  const Span out[2] = {{O, tok * Hv * dv * es}, {S_final, sb}};
  if (int r = check_spans(in, 7, out, 2, 1, 4)) return r;
  return hip_status(gdn::launch_linear_step(Q, K, V, g, g_per_token != 0, S0, O, S_final, slots,
                                            slots ? n_states : nseq, cu_seqlens, nseq, T, Hk, Hv,
                                            dk, dv, scale, dtype, (hipStream_t)stream));
}

int gdn_linear_forward_workspace(int nseq, int T, int Hk, int Hv, int dk, int dv, int packed,
                                 int dtype, int64_t* bytes) {
  if (!bytes) return GDN_ERR_NULL;
  gdn::LinArgs a{};
  if (int r = set_sizes(a, nullptr, packed != 0, nseq, T, Hk, Hv, dk, dv, false, dtype))
    return r;
  *bytes = 4 * gdn::lin_workspace(a, false, nullptr);
  return GDN_OK;
}

int gdn_linear_forward(const void* Q, const void* K, const void* V, const float* g,
                       int g_per_token, const float* S0, void* O, float* S_final, void* workspace,
                       int64_t workspace_bytes, const int32_t* cu_seqlens, int nseq, int T, int Hk,
                       int Hv, int dk, int dv, float scale, int dtype, void* stream) {
  gdn::LinArgs a{};
  if (int r = set_sizes(a, cu_seqlens, cu_seqlens != nullptr, nseq, T, Hk, Hv, dk, dv, false,
                        dtype))
    return r;
  if (!rows_fit(T, Hk, Hv, dk, dv, dtype, 1)) return GDN_ERR_SHAPE;
  if ((int64_t)nseq * Hv == 0) return GDN_OK;
  const int64_t tok = a.q.tokens(), es = esize(dtype);
  int64_t need = 4 * gdn::lin_workspace(a, false, nullptr);
  if (tok > 0) {
    if (!Q || !K || !V || !g || !O || (need && !workspace)) return GDN_ERR_NULL;
    if (workspace_bytes < need) return GDN_ERR_WORKSPACE;
  } else {
    Q = K = V = nullptr, g = nullptr, O = nullptr;
  }
  if (!need) workspace = nullptr;
  const int64_t sb = (int64_t)nseq * Hv * dk * dv * 4;
  const Span in[6] = {{Q, tok * Hk * dk * es},
                      {K, tok * Hk * dk * es},
                      {V, tok * Hv * dv * es},
                      {g, (g_per_token ? tok : 1) * Hv * 4},
                      {S0, sb},
                      {cu_seqlens, 4ll * (nseq + 1)}};
  const Span out[3] = {{O, tok * Hv * dv * es}, {S_final, sb}, {workspace, need}};
  if (int r = check_spans(in, 6, out, 3, 1, 4)) return r;
  a.Q = Q, a.K = K, a.V = V, a.g = g, a.S0 = S0, a.O = O, a.Sf = S_final;
  a.per_token = g_per_token != 0, a.scale = scale;
  gdn::lin_workspace(a, false, (float*)workspace);
  return hip_status(gdn::launch_linear_forward(a, dtype, (hipStream_t)stream));
}

int gdn_linear_backward_workspace(int nseq, int T, int Hk, int Hv, int dk, int dv, int packed,
                                  int dtype, int64_t* bytes) {
  if (!bytes) return GDN_ERR_NULL;
  gdn::LinArgs a{};
  if (int r = set_sizes(a, nullptr, packed != 0, nseq, T, Hk, Hv, dk, dv, true, dtype)) return r;
  a.want_dg = true;
  *bytes = 4 * gdn::lin_workspace(a, true, nullptr);
  return GDN_OK;
}

int gdn_linear_backward(const void* Q, const void* K, const void* V, const float* g,
                        int g_per_token, const void* dO, const float* S0, const float* dS_final,
                        void* dQ, void* dK, void* dV, float* dg, float* dS0, void* workspace,
                        int64_t workspace_bytes, const int32_t* cu_seqlens, int nseq, int T,
                        int Hk, int Hv, int dk, int dv, float scale, int dtype, void* stream) {
  gdn::LinArgs a{};
  if (int r = set_sizes(a, cu_seqlens, cu_seqlens != nullptr, nseq, T, Hk, Hv, dk, dv, true,
                        dtype))
    return r;
  if (!rows_fit(T, Hk, Hv, dk, dv, GDN_F32, 16)) return GDN_ERR_SHAPE;
  if (Hv == 0 || (nseq == 0 && (g_per_token || !dg))) return GDN_OK;
  const int64_t tok = a.q.tokens(), es = esize(dtype);
  a.per_token = g_per_token != 0, a.want_dg = dg != nullptr, a.scale = scale;
  int64_t need = 4 * gdn::lin_workspace(a, true, nullptr);
  if (tok > 0) {
    if (!Q || !K || !V || !g || !dO || !dQ || !dK || !dV || (need && !workspace))
      return GDN_ERR_NULL;
    if (workspace_bytes < need) return GDN_ERR_WORKSPACE;
  } else {
    Q = K = V = dO = nullptr, g = nullptr, dQ = dK = dV = nullptr;
    if (a.per_token) dg = nullptr, a.want_dg = false;
    need = 0;
  }
  if (!need) workspace = nullptr;
  const int64_t kb = tok * Hk * dk * es, vb = tok * Hv * dv * es;
  const int64_t gb = (g_per_token ? tok : 1) * Hv * 4, sb = (int64_t)nseq * Hv * dk * dv * 4;
  const Span in[8] = {{Q, kb},  {K, kb},  {V, vb},         {g, gb},
                      {dO, vb}, {S0, sb}, {dS_final, sb}, {cu_seqlens, 4ll * (nseq + 1)}};
  const Span out[6] = {{dQ, kb}, {dK, kb}, {dV, vb}, {dg, gb}, {dS0, sb}, {workspace, need}};
  if (int r = check_spans(in, 8, out, 6)) return r;
  a.Q = Q, a.K = K, a.V = V, a.dO = dO, a.g = g, a.S0 = S0, a.dSf = dS_final;
  a.dQ = dQ, a.dK = dK, a.dV = dV, a.dg = dg, a.dS0 = dS0;
  gdn::lin_workspace(a, true, (float*)workspace);
  return hip_status(gdn::launch_linear_backward(a, dtype, (hipStream_t)stream));
}

namespace {
constexpr int64_t kMostValues = 1ll << 48;  // of a map; no memory holds as many
int check_group(int64_t N, int S, int C, int G, int dtype) {
  if (N < 0 || N > 0x7fffffffLL || S < 1 || S > 1 << 30 || C < 1 || C > 65536 || G < 1 || C % G)
    return GDN_ERR_SHAPE;
  if (N > 0 && S > kMostValues / C / N) return GDN_ERR_SHAPE;
  if (!fdtype(dtype)) return GDN_ERR_DTYPE;
  return GDN_OK;
}
}  // namespace

int gdn_group_norm_forward_workspace(int64_t N, int S, int C, int G, int dtype, int64_t* bytes) {
  if (!bytes) return GDN_ERR_NULL;
  if (int r = check_group(N, S, C, G, dtype)) return r;
  *bytes = 4 * gdn::group_forward_workspace(N, S, G, C / G, dtype);
  return GDN_OK;
}

int gdn_group_norm_forward(const void* x, const void* w, const void* b, const void* z, void* y,
                           float* mean, float* rstd, void* workspace, int64_t workspace_bytes,
                           int64_t N, int S, int C, int G, float eps, int act, int dtype,
                           int w_dtype, void* stream) {
  if (int r = check_group(N, S, C, G, dtype)) return r;
  if (!fdtype(w_dtype)) return GDN_ERR_DTYPE;
  if ((act != GDN_ACT_NONE && act != GDN_ACT_SILU) || !(eps >= 0.f)) return GDN_ERR_PARAM;
  if (!grid_ok(gdn::group_forward_blocks(N, S, G, C / G, dtype), 256)) return GDN_ERR_SHAPE;
  if (N == 0) return GDN_OK;
  if (!x || !y) return GDN_ERR_NULL;
  const int64_t need = 4 * gdn::group_forward_workspace(N, S, G, C / G, dtype);
  if (need && !workspace) return GDN_ERR_NULL;
  if (workspace_bytes < need) return GDN_ERR_WORKSPACE;
  if (!need) workspace = nullptr;
  const int64_t n = N * S * C * esize(dtype), wb = (int64_t)C * esize(w_dtype), sb = N * G * 4;
  const Span in[4] = {{x, n}, {w, wb}, {b, wb}, {z, n}};
  const Span out[4] = {{y, n}, {mean, sb}, {rstd, sb}, {workspace, need}};
  if (int r = check_spans(in, 4, out, 4)) return r;
  gdn::GroupArgs a{};
  a.x = x, a.w = w, a.b = b, a.z = z, a.out = y, a.mean = mean, a.rstd = rstd;
  a.ws = (float*)workspace, a.N = N, a.S = S, a.G = G, a.Cg = C / G, a.C = C, a.eps = eps;
  a.act = act == GDN_ACT_SILU, a.wbf = w_dtype == GDN_BF16;
  return hip_status(gdn::launch_group_forward(a, dtype, (hipStream_t)stream));
}

int gdn_group_norm_backward_workspace(int64_t N, int S, int C, int G, int dtype, int64_t* bytes) {
  if (!bytes) return GDN_ERR_NULL;
  if (int r = check_group(N, S, C, G, dtype)) return r;
  *bytes = 4 * gdn::group_backward_workspace(N, S, G, C / G, dtype);
  return GDN_OK;
}

int gdn_group_norm_backward(const void* dy, const void* x, const void* w, const void* b,
                            const void* z, const float* mean, const float* rstd, void* dx,
                            float* dw, float* db, void* dz, void* workspace,
                            int64_t workspace_bytes, int64_t N, int S, int C, int G, int act,
                            int dtype, int w_dtype, void* stream) {
  if (int r = check_group(N, S, C, G, dtype)) return r;
  if (!fdtype(w_dtype)) return GDN_ERR_DTYPE;
  if (act != GDN_ACT_NONE && act != GDN_ACT_SILU) return GDN_ERR_PARAM;
  if (!grid_ok(gdn::group_backward_blocks(N, S, G, C / G, dtype), 256)) return GDN_ERR_SHAPE;
  if (N == 0 && !dw && !db) return GDN_OK;
  int64_t need = 4 * gdn::group_backward_workspace(N, S, G, C / G, dtype, dw || db);
  if (N > 0) {
    if (!dy || !x || !mean || !rstd || !dx || (z && !dz) || (need && !workspace))
      return GDN_ERR_NULL;
    if (workspace_bytes < need) return GDN_ERR_WORKSPACE;
  } else {
    need = 0;
  }
  if (!need) workspace = nullptr;
  if (!z) dz = nullptr;
  const int64_t n = N * S * C * esize(dtype), wb = (int64_t)C * esize(w_dtype), sb = N * G * 4;
  const Span in[7] = {{dy, n}, {x, n}, {w, wb}, {b, wb}, {z, n}, {mean, sb}, {rstd, sb}};
  const Span out[5] = {{dx, n}, {dw, 4ll * C}, {db, 4ll * C}, {dz, n}, {workspace, need}};
  if (int r = check_spans(in, 7, out, 5)) return r;
  gdn::GroupArgs a{};
  a.dy = dy, a.x = x, a.w = w, a.b = b, a.z = z, a.mean_in = mean, a.rstd_in = rstd;
  a.out = dx, a.dz = dz, a.dw = dw, a.db = db, a.ws = (float*)workspace;
  a.N = N, a.S = S, a.G = G, a.Cg = C / G, a.C = C;
  a.act = act == GDN_ACT_SILU, a.wbf = w_dtype == GDN_BF16;
  return hip_status(gdn::launch_group_backward(a, dtype, (hipStream_t)stream));
}

}  // extern "C"
