// linear.hpp -- linear attention with a decay for each head: what its launches share
// (linear.hip the chunked form and its gradients, linear_step.hip the recurrent form).
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

namespace gdn {

// Tokens a chunk, the step of a walk.
constexpr int LC = 64;

// Sequences, and how they are cut into segments of `seg` tokens (a multiple of LC), which
// have slots: sequence s has those from base(s).  Packed sequences: base(s) =
// cu[s] / seg + s needs no table, and base(s + 1) - base(s) is at least the sequence's
// segments.  A sequence with an offset out of range, or that ends before it begins, is empty.
struct LinSeqs {
  const int* cu;  // nseq + 1 token offsets, or null
  int nseq, T;    // T: tokens of each sequence, or of all where cu is given
  int seg, nseg;  // nseg: segments a sequence (cu null)

  // (no sequences have neither, whatever T: cu holds one offset then)
  __host__ __device__ int64_t slots() const {
    return cu ? (nseq ? (int64_t)T / seg + nseq : 0) : (int64_t)nseq * nseg;
  }
  __host__ __device__ int64_t tokens() const {
    return cu ? (nseq ? T : 0) : (int64_t)nseq * T;
  }
  __host__ __device__ int segments(int len) const { return len > 0 ? (len - 1) / seg + 1 : 0; }
  __device__ void at(int s, int64_t& t0, int64_t& base, int& len) const {
    if (cu) {
      const int b = cu[s], e = cu[s + 1];
      const bool ok = b >= 0 && e >= b && e <= T;
      t0 = ok ? b : 0;
      len = ok ? e - b : 0;
      base = t0 / seg + s;
    } else {
      t0 = (int64_t)s * T;
      len = T;
      base = (int64_t)s * nseg;
    }
  }
  // the sequence that may have a slot: the last one that begins in range with base <= slot.
  // The whole wave calls.
  __device__ int find(uint32_t slot) const {
    if (!cu) return (int)(slot / (uint32_t)nseg);
    int lo = 0, hi = nseq;
    while (hi - lo > 64) {  // an offset out of range says nothing: the next one in range does
      const int mid = (lo + hi) >> 1;
      int i = mid, b = cu[i];
      while ((b < 0 || b > T) && ++i < hi) b = cu[i];
      if (i < hi && (int64_t)b / seg + i <= slot) lo = i; else hi = mid;
    }
    const int i = lo + (int)(threadIdx.x & 63);
    bool before = false;
    if (i < hi) {
      const int b = cu[i];
      before = b >= 0 && b <= T && (int64_t)b / seg + i <= slot;
    }
    const uint64_t mask = __ballot(before);
    return mask ? lo + 63 - __builtin_clzll(mask) : lo;
  }
};

// One call of the forward or backward pass.
struct LinArgs {
  LinSeqs q;
  const void *Q, *K, *V, *dO;
  const float *g, *S0, *dSf;  // g: [Hv], or [tokens, Hv] with per_token
  bool per_token, want_dg;
  void *O, *dQ, *dK, *dV;
  float *Sf, *dS0, *dg;
  int Hk, Hv, dk, dv;
  float scale;
  // workspace, each null where it is not needed (U, R, dec: every sequence is one segment; acc_q,
  // acc_k: one value head a key head; the others: no dg)
  float *U, *R;           // [slots, Hv, dk, dv]: states entering, their gradients leaving
  float* dec;             // [slots, Hv]: decay over a segment
  float *rows_q, *rows_k;  // [Hv, tokens]: what dg takes of each token (linear.hip)
  float *anchor, *part;   // [slots, Hv]: X of a segment's first chunk; sums of dg
  float *acc_q, *acc_k;   // [tokens, Hk, dk]: sums of dQ, dK over a group's first heads
};

// Tokens a segment for these sizes.
int lin_segment(int nseq, int T, int Hk, int Hv, int dk, int dv, bool packed, bool backward,
                bool fp32);
// Floats of workspace; fills in the pointers where ws is given.
int64_t lin_workspace(LinArgs& a, bool backward, float* ws);

// Value columns a wave of the recurrent form takes; a workgroup has four waves.
constexpr int kStepColumns = 32;

hipError_t launch_linear_forward(const LinArgs& a, int dtype, hipStream_t st);
hipError_t launch_linear_backward(const LinArgs& a, int dtype, hipStream_t st);
hipError_t launch_linear_step(const void* Q, const void* K, const void* V, const float* g,
                              bool per_token, const float* S0, void* O, float* Sfin,
                              const int* slots, int n_states, const int* cu, int nseq, int T,
                              int Hk, int Hv, int dk, int dv, float scale, int dtype,
                              hipStream_t st);

}  // namespace gdn
