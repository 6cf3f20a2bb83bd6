/*
 * gdnlinear.h -- C ABI of linear attention with a decay for each head (the
 * layer of gdninv.h and gdnlayer.h without the delta rule's correction), for
 * training and serving, and of group norm, channels last.  Same library
 * (libgdninv.so), status codes, dtypes and conventions as gdninv.h: device
 * pointers owned by the caller, 16-byte aligned, dense and row-major; work is
 * only enqueued on `stream`; arguments are validated before anything is
 * enqueued; no memory is allocated.
 *
 * Shared key heads.  Q and K hold Hk heads and V, O and the states Hv heads,
 * Hv a multiple of Hk: value head h reads key head h / (Hv / Hk).
 */
#ifndef GDNLINEAR_H
#define GDNLINEAR_H

#include "gdninv.h"

#ifdef __cplusplus
extern "C" {
#endif

/* Linear attention with decay: per sequence and value head, with the [dk, dv]
 * state S in fp32,
 *   S_t = e^{g_t} S_{t-1} + k_t v_t^T,   o_t = scale S_t^T q_t.
 * g is a log-decay (<= 0 for a decay): of each token and head, [tokens, Hv]
 * fp32, where g_per_token is set, else one of each head, [Hv].  -inf forgets
 * everything before the token.
 *
 * cu_seqlens NULL: nseq sequences of T tokens, Q, K [nseq, T, Hk, dk], V, O
 * [nseq, T, Hv, dv].  Otherwise packed sequences (nseq + 1 int32 token offsets
 * on the device, non-decreasing, within 0 .. T): Q, K [T, Hk, dk] and so on; a
 * sequence with an offset out of range, or that ends before it begins, is taken
 * as empty, whichever of the sequences it is, and tokens outside every sequence
 * get no output.  Offsets within range have to be non-decreasing: nothing
 * outside the arrays is touched where they are not, but the results are
 * undefined.  Without sequences (nseq = 0) nothing is read, and nothing is
 * written but the gradients of the heads' decays, 0.
 *
 * dk, dv in {64, 128}; dtype GDN_F32 or GDN_BF16; T >= 0.  Sums, states and
 * decays are fp32 (the sums of g 64-bit) whatever the dtype, O rounds once. */

/* Whole sequences, chunk by chunk.  S0 (nullable: zero states) and S_final
 * (nullable: not written) are [nseq, Hv, dk, dv] fp32; S_final may be S0 itself
 * but must not overlap it otherwise.  An empty sequence keeps its state.  The
 * rows of all heads of 64 tokens (of T where that is less) of Q and of V hold
 * 4 GiB at most.
 * With bf16 inputs the states, the products q . k under the decay and the values
 * under the decay enter products as sums of three bf16 terms (2^-24 of each).
 * A value that is not finite makes what it reaches not finite either (an
 * infinity NaN), and may do so to other tokens of its 64, counted from the
 * sequence's first; it reaches no other sequence and no other value head that
 * does not read it.  A token reaches those after it as far as the decay between
 * them is not 0 in fp32 (e^-104); whether a value that is not finite reaches
 * further is not defined.
 * workspace: at least gdn_linear_forward_workspace() bytes (may be NULL where
 * that is 0), contents undefined on return.  One launch, or three where a
 * sequence is cut into segments. */
int gdn_linear_forward(const void* Q, const void* K, const void* V, const float* g,
                       int g_per_token, const float* S0, void* O, float* S_final, void* workspace,
                       int64_t workspace_bytes, const int32_t* cu_seqlens, int nseq, int T, int Hk,
                       int Hv, int dk, int dv, float scale, int dtype, void* stream);

/* Workspace bytes for nseq sequences of T tokens (packed = 0), or of T tokens
 * in all (packed = 1). */
int gdn_linear_forward_workspace(int nseq, int T, int Hk, int Hv, int dk, int dv, int packed,
                                 int dtype, int64_t* bytes);

/* Gradients of gdn_linear_forward: from dO and, where given, dS_final (the
 * gradient of the final states; NULL: zero) those of Q, K, V and, where asked
 * for (nullable), of g (fp32, as given: [tokens, Hv] or [Hv]) and of S0.
 * Nothing of the forward pass is kept for it.  The gradients of a key head sum
 * over its group of value heads, those of a head's decay over all its tokens.
 * Everything is formed in fp32 or sums of bf16 terms that make it up and
 * rounded once at the end, in a fixed order: the same call gives the same bits.
 * The rows of all heads of 64 tokens (of T where that is less, of 16 at least)
 * hold 2^30 values at most.
 * A value that is not finite reaches what it does in the forward pass, and
 * through dQ and dK the key head's other gradients; dg of a token reaches from
 * the tokens after it.
 * workspace: at least gdn_linear_backward_workspace() bytes. */
int gdn_linear_backward(const void* Q, const void* K, const void* V, const float* g,
                        int g_per_token, const void* dO, const float* S0, const float* dS_final,
                        void* dQ, void* dK, void* dV, float* dg, float* dS0, void* workspace,
                        int64_t workspace_bytes, const int32_t* cu_seqlens, int nseq, int T,
                        int Hk, int Hv, int dk, int dv, float scale, int dtype, void* stream);

/* Workspace bytes of gdn_linear_backward, wanting every gradient. */
int gdn_linear_backward_workspace(int nseq, int T, int Hk, int Hv, int dk, int dv, int packed,
                                  int dtype, int64_t* bytes);

/* The same token by token, for decoding, all of it in fp32 (O rounds once).
 * S0 (nullable: zero states) and S_final (nullable: not written) hold n_states
 * states [n_states, Hv, dk, dv] fp32; S_final may be S0 itself (updated in
 * place) but must not overlap it otherwise.  slots (nullable: sequence s has
 * state s, n_states >= nseq): int32 state index of every sequence, on the
 * device; an index outside 0 .. n_states - 1 marks a padded sequence, whose
 * rows of O are written as zeros and which touches no state.  Two sequences
 * must not share a slot when S_final is written.  A sequence without tokens
 * copies its state (nothing to do in place). */
int gdn_linear_recurrent(const void* Q, const void* K, const void* V, const float* g,
                         int g_per_token, const float* S0, void* O, float* S_final,
                         const int32_t* slots, int n_states, const int32_t* cu_seqlens, int nseq,
                         int T, int Hk, int Hv, int dk, int dv, float scale, int dtype,
                         void* stream);

enum gdn_act { GDN_ACT_NONE = 0, GDN_ACT_SILU = 1 };

/* Group norm, channels last: x [N, S, C], the C channels in G groups of C / G
 * neighbours, mean and rstd of each (n, group) over its S positions and C / G
 * channels:
 *   n = (x - mean) rstd w + b,  rstd = (mean((x - mean)^2) + eps)^-1/2,
 *   y = act(n) silu(z),  act(n) = n or silu(n),  silu(t) = t / (1 + e^-t).
 * x, z, y [N, S, C] in dtype (GDN_F32 or GDN_BF16); w, b [C] in w_dtype.  w, b
 * and z may be NULL (factor 1, no bias, no gate).  mean, rstd [N, G] fp32, each
 * nullable: what the backward pass takes.  Statistics and products are fp32; y
 * rounds once.  One group a head and S = 1 is the norm of a layer's heads with
 * weights of their own.
 * 0 <= N < 2^31, 1 <= S <= 2^30, 1 <= C <= 65536, N S C <= 2^48, any sizes and
 * row alignment.  Groups of more than 256 pieces (of 16 bytes; of a value or two
 * where a group's channels do not fill such pieces), of more than 1024 where
 * S = 1, and in the backward pass all with S > 1, are read twice: up to 2^24
 * workgroups, one for every 256 pieces of the C channels and each n.
 * workspace: at least gdn_group_norm_forward_workspace() bytes (may be NULL
 * where that is 0). */
int gdn_group_norm_forward(const void* x, const void* w, const void* b, const void* z, void* y,
                           float* mean, float* rstd, void* workspace, int64_t workspace_bytes,
                           int64_t N, int S, int C, int G, float eps, int act, int dtype,
                           int w_dtype, void* stream);

int gdn_group_norm_forward_workspace(int64_t N, int S, int C, int G, int dtype, int64_t* bytes);

/* Gradients of gdn_group_norm_forward from dy [N, S, C]: dx and, where z is
 * given, dz [N, S, C] in dtype; dw, db [C] fp32, summed over n and positions
 * (each nullable: not formed).  mean and rstd as the forward pass wrote them.
 * The sums are taken in a fixed order: the same call gives the same bits.
 * workspace: at least gdn_group_norm_backward_workspace() bytes; groups that are
 * read once take none (NULL) where neither dw nor db is formed. */
int gdn_group_norm_backward(const void* dy, const void* x, const void* w, const void* b,
                            const void* z, const float* mean, const float* rstd, void* dx,
                            float* dw, float* db, void* dz, void* workspace,
                            int64_t workspace_bytes, int64_t N, int S, int C, int G, int act,
                            int dtype, int w_dtype, void* stream);

int gdn_group_norm_backward_workspace(int64_t N, int S, int C, int G, int dtype, int64_t* bytes);

#ifdef __cplusplus
}
#endif

#endif /* GDNLINEAR_H */
