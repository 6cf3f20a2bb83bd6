// api_layer.cpp -- the extern "C" boundary declared in include/gdnlayer.h.
// Validates every argument before anything is enqueued, then dispatches to
// the launchers.  Holds no state.
#include "gdnlayer.h"

#include <stdint.h>

#include <algorithm>

#include "checks.hpp"
#include "layer.hpp"

namespace {

using namespace gdn::checks;

// a device array of the call: its address and bytes
struct Span {
  const void* p;
  int64_t bytes;
};

// every array aligned; no output overlaps an input or another output, but for
// output same_out and input same_in where these are one array
int check_spans(const Span* in, int ni, const Span* out, int no, int same_out = -1,
                int same_in = -1) {
  for (int i = 0; i < ni; ++i)
    if (in[i].p && !aligned(in[i].p)) return GDN_ERR_ALIGN;
  for (int o = 0; o < no; ++o)
    if (out[o].p && !aligned(out[o].p)) return GDN_ERR_ALIGN;
  for (int o = 0; o < no; ++o) {
    for (int i = 0; i < ni; ++i) {
      if (o == same_out && i == same_in && out[o].p == in[i].p) continue;
      if (overlap(out[o].p, out[o].bytes, in[i].p, in[i].bytes)) return GDN_ERR_ALIAS;
    }
    for (int q = o + 1; q < no; ++q)
      if (overlap(out[o].p, out[o].bytes, out[q].p, out[q].bytes)) return GDN_ERR_ALIAS;
  }
  return GDN_OK;
}

bool valid_heads(int Hk, int Hv) { return Hk >= 0 && Hv >= 0 && (Hk ? Hv % Hk == 0 : Hv == 0); }

}  // namespace

extern "C" {

int gdn_recurrent_forward(const void* Q, const void* K, const void* V, const float* beta,
                          const float* g, const float* S0, void* O, float* S_final,
                          const int32_t* slots, int n_states, const int32_t* cu_seqlens, int nseq,
                          int T, int Hk, int Hv, int dk, int dv, float scale, int dtype,
                          void* stream) {
  if (nseq < 0 || T < 0 || n_states < 0 || !valid_heads(Hk, Hv)) return GDN_ERR_SHAPE;
  if (!valid_d(dk) || !valid_d(dv)) return GDN_ERR_SHAPE;
  if (!slots && n_states < nseq && (S0 || S_final)) return GDN_ERR_SHAPE;
  if (!grid_ok(((int64_t)nseq * Hv * (dv / 32) + 3) / 4, 256)) return GDN_ERR_SHAPE;
  if (!fdtype(dtype)) return GDN_ERR_DTYPE;
  if ((int64_t)nseq * Hv == 0) return GDN_OK;
  const int64_t tok = cu_seqlens ? (int64_t)T : (int64_t)nseq * T, es = esize(dtype);
  if (tok > 0 && (!Q || !K || !V || !beta || !g || !O)) return GDN_ERR_NULL;
  if (tok == 0) Q = K = V = nullptr, beta = g = nullptr, O = nullptr;
  const int64_t sb = (int64_t)(slots ? n_states : nseq) * Hv * dk * dv * 4;
  const Span in[8] = {{Q, tok * Hk * dk * es}, {K, tok * Hk * dk * es}, {V, tok * Hv * dv * es},
                      {beta, tok * Hv * 4},    {g, tok * Hv * 4},       {S0, sb},
                      {slots, 4ll * nseq},     {cu_seqlens, 4ll * (nseq + 1)}};
  const Span out[2] = {{O, tok * Hv * dv * es}, {S_final, sb}};
  if (int r = check_spans(in, 8, out, 2, 1, 5)) return r;
  return hip_status(gdn::launch_recurrent(Q, K, V, beta, g, S0, O, S_final, slots,
                                          slots ? n_states : nseq, cu_seqlens, nseq, T, Hk, Hv,
                                          dk, dv, scale, dtype, (hipStream_t)stream));
}

int gdn_chunk_backward_workspace(int nseq, int L, int Hv, int dk, int dv, int packed,
                                 int64_t* bytes) {
  if (!bytes) return GDN_ERR_NULL;
  if (nseq < 0 || L < 0 || Hv < 0 || !valid_d(dk) || !valid_d(dv)) return GDN_ERR_SHAPE;
  const int64_t slots = L > 0 && nseq > 0 ? gdn::backward_slots(nseq, L, packed != 0) : 0;
  // (the per-chunk launches' workgroups have 512 work items at most)
  if (Hv > 0 && (!grid_ok(slots, 512) || !grid_ok(slots * Hv, 512))) return GDN_ERR_SHAPE;
  *bytes = slots * Hv * gdn::backward_tile_bytes(dk, dv);
  return GDN_OK;
}

namespace {
int backward(const void* Q, const void* K, const void* V, const float* beta, const float* g,
             const void* dO, const float* S0, const float* dS_final, void* dQ, void* dK, void* dV,
             float* dbeta, float* dg, float* dS0, void* workspace, int64_t workspace_bytes,
             const int32_t* cu, bool packed, int nseq, int L, int Hk, int Hv, int dk, int dv,
             int C, float scale, int dtype, void* stream) {
  if (!valid_heads(Hk, Hv)) return GDN_ERR_SHAPE;
  if (!(C == 16 || C == 32 || C == 64)) return C == 128 ? GDN_ERR_UNSUPPORTED : GDN_ERR_SHAPE;
  int64_t need = 0;
  if (int r = gdn_chunk_backward_workspace(nseq, L, Hv, dk, dv, packed, &need)) return r;
  if (!grid_ok(((int64_t)nseq * Hv + 7) / 8 * 8 * (dv / 16), 512)) return GDN_ERR_SHAPE;
  if (!fdtype(dtype)) return GDN_ERR_DTYPE;
  if (packed && L > 0 && dtype == GDN_BF16 &&
      !grid_ok(gdn::packed_walk_groups(nseq, Hv, dv), 512))
    return GDN_ERR_SHAPE;
  // (rows of a chunk of 64 tokens lie at 32-bit byte offsets from its first)
  const int64_t tok = packed ? (int64_t)L : (int64_t)nseq * L, es = esize(dtype);
  const int64_t row = std::max((int64_t)Hk * dk, (int64_t)Hv * dv) * es;
  if (std::min(L, 64) * row > 1ll << 32) return GDN_ERR_SHAPE;
  if ((int64_t)nseq * Hv == 0) return GDN_OK;
  if (packed && !cu) return GDN_ERR_NULL;
  if (tok > 0) {
    if (!Q || !K || !V || !beta || !g || !dO || !dQ || !dK || !dV || !dbeta || !dg || !workspace)
      return GDN_ERR_NULL;
    if (workspace_bytes < need) return GDN_ERR_WORKSPACE;
  } else {
    Q = K = V = dO = nullptr, beta = g = nullptr, dQ = dK = dV = workspace = nullptr;
    dbeta = dg = nullptr;
  }
  const int64_t kb = tok * Hk * dk * es, vb = tok * Hv * dv * es, bb = tok * Hv * 4;
  const int64_t sb = (int64_t)nseq * Hv * dk * dv * 4;
  const Span in[9] = {{Q, kb},  {K, kb},   {V, vb},         {beta, bb},          {g, bb},
                      {dO, vb}, {S0, sb}, {dS_final, sb}, {cu, 4ll * (nseq + 1)}};
  const Span out[7] = {{dQ, kb}, {dK, kb},  {dV, vb},          {dbeta, bb},
                       {dg, bb}, {dS0, sb}, {workspace, need}};
  if (int r = check_spans(in, 9, out, 7)) return r;
  return hip_status(gdn::launch_backward(Q, K, V, beta, g, dO, S0, dS_final, dQ, dK, dV, dbeta, dg,
                                         dS0, (float*)workspace, cu, nseq, L, Hk, Hv, dk, dv, C,
                                         scale, dtype, (hipStream_t)stream));
}
}  // namespace

int gdn_chunk_backward(const void* Q, const void* K, const void* V, const float* beta,
                       const float* g, const void* dO, const float* S0, const float* dS_final,
                       void* dQ, void* dK, void* dV, float* dbeta, float* dg, float* dS0,
                       void* workspace, int64_t workspace_bytes, int B, int L, int Hk, int Hv,
                       int dk, int dv, int C, float scale, int dtype, void* stream) {
  return backward(Q, K, V, beta, g, dO, S0, dS_final, dQ, dK, dV, dbeta, dg, dS0, workspace,
                  workspace_bytes, nullptr, false, B, L, Hk, Hv, dk, dv, C, scale, dtype, stream);
}

int gdn_chunk_backward_varlen(const void* Q, const void* K, const void* V, const float* beta,
                              const float* g, const void* dO, const float* S0,
                              const float* dS_final, void* dQ, void* dK, void* dV, float* dbeta,
                              float* dg, float* dS0, void* workspace, int64_t workspace_bytes,
                              const int32_t* cu_seqlens, int nseq, int T, int Hk, int Hv, int dk,
                              int dv, int C, float scale, int dtype, void* stream) {
  return backward(Q, K, V, beta, g, dO, S0, dS_final, dQ, dK, dV, dbeta, dg, dS0, workspace,
                  workspace_bytes, cu_seqlens, true, nseq, T, Hk, Hv, dk, dv, C, scale, dtype,
                  stream);
}

namespace {
int check_norm(int64_t rows, int D, int kind, int dtype, int w_dtype) {
  if (rows < 0 || rows > 0x7fffffffLL || D < 1 || D > 65536) return GDN_ERR_SHAPE;
  if (kind != GDN_NORM_LAYER && kind != GDN_NORM_RMS) return GDN_ERR_PARAM;
  if (!fdtype(dtype) || !fdtype(w_dtype)) return GDN_ERR_DTYPE;
  return GDN_OK;
}
}  // namespace

int gdn_norm_forward(const void* x, const void* w, const void* b, const void* z, void* y,
                     float* mean, float* rstd, int64_t rows, int D, float eps, int kind,
                     int dtype, int w_dtype, void* stream) {
  if (int r = check_norm(rows, D, kind, dtype, w_dtype)) return r;
  if (!(eps >= 0.f)) return GDN_ERR_PARAM;
  if (rows == 0) return GDN_OK;
  if (!x || !y) return GDN_ERR_NULL;
  const bool rms = kind == GDN_NORM_RMS;
  if (rms) mean = nullptr;
  const int64_t n = rows * D * esize(dtype), wb = (int64_t)D * esize(w_dtype);
  const Span in[4] = {{x, n}, {w, wb}, {b, wb}, {z, n}};
  const Span out[3] = {{y, n}, {mean, rows * 4}, {rstd, rows * 4}};
  if (int r = check_spans(in, 4, out, 3)) return r;
  return hip_status(gdn::launch_norm_forward(x, w, b, z, y, mean, rstd, rows, D, eps, rms, dtype,
                                             w_dtype, (hipStream_t)stream));
}

int gdn_norm_backward_workspace(int64_t rows, int D, int64_t* bytes) {
  if (!bytes) return GDN_ERR_NULL;
  if (int r = check_norm(rows, D, GDN_NORM_RMS, GDN_F32, GDN_F32)) return r;
  *bytes = (int64_t)gdn::norm_backward_parts(rows) * D * 2 * 4;
  return GDN_OK;
}

int gdn_norm_backward(const void* dy, const void* x, const void* w, const void* b, const void* z,
                      const float* mean, const float* rstd, void* dx, float* dw, float* db,
                      void* dz, void* workspace, int64_t workspace_bytes, int64_t rows, int D,
                      int kind, int dtype, int w_dtype, void* stream) {
  if (int r = check_norm(rows, D, kind, dtype, w_dtype)) return r;
  const bool rms = kind == GDN_NORM_RMS;
  int64_t need = 0;
  if (int r = gdn_norm_backward_workspace(rows, D, &need)) return r;
  if (!dw && !db) need = 0;
  if (rows > 0) {
    if (!dy || !x || !rstd || !dx || (!rms && !mean) || (z && !dz) || (need && !workspace))
      return GDN_ERR_NULL;
    if (workspace_bytes < need) return GDN_ERR_WORKSPACE;
  }
  if (rms) mean = nullptr;
  if (!z) dz = nullptr;
  if (!need) workspace = nullptr;
  const int64_t n = rows * D * esize(dtype), wb = (int64_t)D * esize(w_dtype);
  const Span in[7] = {{dy, n}, {x, n}, {w, wb}, {b, wb}, {z, n}, {mean, rows * 4}, {rstd, rows * 4}};
  const Span out[5] = {{dx, n}, {dw, 4ll * D}, {db, 4ll * D}, {dz, n}, {workspace, need}};
  if (int r = check_spans(in, 7, out, 5)) return r;
  return hip_status(gdn::launch_norm_backward(dy, x, w, b, z, mean, rstd, dx, dw, db, dz,
                                              (float*)workspace, rows, D, rms, dtype, w_dtype,
                                              (hipStream_t)stream));
}

}  // extern "C"
