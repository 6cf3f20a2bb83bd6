/*
 * gdnlayer.h -- C ABI of the operators that train and serve a Gated DeltaNet
 * layer around the chunk-wise forward of gdninv.h: the recurrent (token by
 * token) form, the chunk-wise backward pass, and the norms of the layer's
 * input and output.  Same library (libgdninv.so), status codes, dtypes and
 * conventions as gdninv.h: device pointers owned by the caller, 16-byte
 * aligned, dense and row-major; work is only enqueued on `stream`; arguments
 * are validated before anything is enqueued; no memory is allocated.
 *
 * Shared key heads.  Q and K hold Hk heads and V, O, beta, g Hv heads, Hv a
 * multiple of Hk: value head h reads key head h / (Hv / Hk).
 */
#ifndef GDNLAYER_H
#define GDNLAYER_H

#include "gdninv.h"

#ifdef __cplusplus
extern "C" {
#endif

/* The gated delta rule token by token, for decoding: per sequence and value
 * head, with the [dk, dv] state S in fp32,
 *   S <- exp(g_t) S,  u = beta_t (v_t - S^T k_t),  S <- S + k_t u^T,
 *   o_t = scale S^T q_t,
 * all of it in fp32 whatever dtype the tensors have (O rounds once).  g is
 * the log-decay of the token itself (not a cumulative sum).
 * cu_seqlens NULL: nseq sequences of T tokens, Q, K [nseq, T, Hk, dk], V, O
 * [nseq, T, Hv, dv], beta, g [nseq, T, Hv] fp32.  Otherwise packed sequences
 * (nseq + 1 int32 token offsets on the device, non-decreasing, within
 * 0 .. T): Q, K [T, Hk, dk] and so on; a sequence whose offsets are out of
 * range is taken as empty, and tokens outside every sequence get no output.
 * S0 (nullable: zero states) and S_final (nullable: not written) hold
 * n_states states [n_states, Hv, dk, dv] fp32; S_final may be S0 itself
 * (updated in place) but must not overlap it otherwise.  slots (nullable:
 * sequence s has state s, n_states >= nseq): int32 state index of every
 * sequence, on the device; an index outside 0 .. n_states - 1 marks a padded
 * sequence, whose rows of O are written as zeros and which touches no state.
 * Two sequences must not share a slot when S_final is written.  A sequence
 * without tokens copies its state (nothing to do in place).  T >= 0;
 * dk, dv in {64, 128}. */
int gdn_recurrent_forward(const void* Q, const void* K, const void* V, const float* beta,
                          const float* g, const float* S0, void* O, float* S_final,
                          const int32_t* slots, int n_states, const int32_t* cu_seqlens, int nseq,
                          int T, int Hk, int Hv, int dk, int dv, float scale, int dtype,
                          void* stream);

/* Gradients of the layer forward gdn_chunk_forward computes with the exact
 * inverse (exact = 1): from dO and, where given, dS_final (the gradient of
 * the final state; NULL: zero) those of Q, K, V, beta, g and S0.  Nothing of
 * the forward pass is kept for it; the states are formed again.
 * Q, K, dQ, dK [B, L, Hk, dk]; V, dO, dV [B, L, Hv, dv] in dtype (GDN_F32 or
 * GDN_BF16); beta, g, dbeta, dg [B, L, Hv] fp32; S0 (NULL: zero states),
 * dS_final, dS0 (nullable: not formed) [B, Hv, dk, dv] fp32.  g is the
 * cumulative log-decay inside chunks of C tokens (C in {16, 32, 64}) from the
 * start of each sequence, as for gdn_chunk_forward, and dg the gradient of g
 * as given; L need not be a multiple of C.  The gradients of a key head sum
 * over its group of value heads.  Everything is formed in fp32 (bf16 inputs
 * enter unrounded) and rounded once at the end, in a fixed order: the same
 * call gives the same bits.
 * A value that is not finite, of the inputs or by overflow on the way, makes
 * what it reaches not finite either, an infinity NaN where bf16 inputs are
 * multiplied (their products with fp32 values run as sums of bf16 terms, the
 * second of which is inf - inf; so do finite ones from 2^128 - 2^119 on).  It
 * reaches no other sequence, and no other value head but through dQ and dK of
 * its key head.
 * workspace: at least gdn_chunk_backward_workspace() bytes, contents
 * undefined on return.  dk, dv in {64, 128}; the rows of all heads of 64 tokens
 * (of L where that is less) of Q and of V hold 4 GiB at most.  Three launches
 * on `stream`. */
int gdn_chunk_backward(const void* Q, const void* K, const void* V, const float* beta,
                       const float* g, const void* dO, const float* S0, const float* dS_final,
                       void* dQ, void* dK, void* dV, float* dbeta, float* dg, float* dS0,
                       void* workspace, int64_t workspace_bytes, int B, int L, int Hk, int Hv,
                       int dk, int dv, int C, float scale, int dtype, void* stream);

/* The same over packed sequences, as gdn_chunk_forward_varlen runs them: the
 * tensors hold T tokens, sequence s those of cu_seqlens[s] .. cu_seqlens[s +
 * 1] - 1 (nseq + 1 int32 offsets on the device, non-decreasing, within
 * 0 .. T); the states are [nseq, Hv, dk, dv].  A sequence with an offset out
 * of range, or ending before it begins, is taken as empty (dS0 = dS_final),
 * whichever of the sequences it is; tokens outside every sequence get no
 * gradients written.  Offsets within range have to be non-decreasing: nothing
 * outside the arrays is touched where they are not, but the gradients are
 * undefined. */
int gdn_chunk_backward_varlen(const void* Q, const void* K, const void* V, const float* beta,
                              const float* g, const void* dO, const float* S0,
                              const float* dS_final, void* dQ, void* dK, void* dV, float* dbeta,
                              float* dg, float* dS0, void* workspace, int64_t workspace_bytes,
                              const int32_t* cu_seqlens, int nseq, int T, int Hk, int Hv, int dk,
                              int dv, int C, float scale, int dtype, void* stream);

/* Workspace bytes of gdn_chunk_backward for nseq = B sequences of L tokens
 * (packed = 0), or of gdn_chunk_backward_varlen for nseq sequences of L = T
 * tokens in all (packed = 1). */
int gdn_chunk_backward_workspace(int nseq, int L, int Hv, int dk, int dv, int packed,
                                 int64_t* bytes);

enum gdn_norm_kind { GDN_NORM_LAYER = 0, GDN_NORM_RMS = 1 };

/* Norm of every row of x [rows, D]:
 *   GDN_NORM_LAYER: xh = (x - mean) rstd, rstd = (mean((x - mean)^2) + eps)^-1/2
 *   GDN_NORM_RMS:   xh = x rstd,          rstd = (mean(x^2) + eps)^-1/2
 *   y = (xh w + b) silu(z),  silu(z) = z / (1 + e^-z).
 * x, z, y [rows, D] in dtype (GDN_F32 or GDN_BF16); w, b [D] in w_dtype.
 * w, b and z may be NULL (factor 1, no bias, no gate).  mean, rstd [rows]
 * fp32, each nullable: what the backward pass takes (mean is not written for
 * GDN_NORM_RMS).  Statistics and products are fp32; y rounds once.
 * 1 <= D <= 65536, any D and any row alignment. */
int gdn_norm_forward(const void* x, const void* w, const void* b, const void* z, void* y,
                     float* mean, float* rstd, int64_t rows, int D, float eps, int kind,
                     int dtype, int w_dtype, void* stream);

/* Gradients of gdn_norm_forward from dy [rows, D]: dx [rows, D] and, where z
 * is given, dz [rows, D] in dtype; dw, db [D] fp32, summed over the rows (each
 * nullable: not formed).  rstd and, for GDN_NORM_LAYER, mean as the forward
 * pass wrote them.  b is read only where z is given (NULL: no bias).
 * workspace: at least gdn_norm_backward_workspace() bytes (may be NULL when
 * that is 0).  The row sums are taken in a fixed order: the same call gives
 * the same bits. */
int gdn_norm_backward(const void* dy, const void* x, const void* w, const void* b, const void* z,
                      const float* mean, const float* rstd, void* dx, float* dw, float* db,
                      void* dz, void* workspace, int64_t workspace_bytes, int64_t rows, int D,
                      int kind, int dtype, int w_dtype, void* stream);

/* Workspace bytes gdn_norm_backward needs for these sizes (wanting both dw
 * and db). */
int gdn_norm_backward_workspace(int64_t rows, int D, int64_t* bytes);

#ifdef __cplusplus
}
#endif

#endif /* GDNLAYER_H */
