// layer.hpp -- host-side launchers of the layer's training and serving
// operators (internal; arguments validated by api_layer.cpp).
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

namespace gdn {

hipError_t launch_recurrent(const void* Q, const void* K, const void* V, const float* beta,
                            const float* g, const float* S0, void* O, float* Sfin,
                            const int* slots, int n_states, const int* cu, int nseq, int T, int Hk,
                            int Hv, int dk, int dv, float scale, int dtype, hipStream_t st);

hipError_t launch_norm_forward(const void* x, const void* w, const void* b, const void* z, void* y,
                               float* mean, float* rstd, int64_t rows, int D, float eps, bool rms,
                               int dtype, int w_dtype, hipStream_t st);
hipError_t launch_norm_backward(const void* dy, const void* x, const void* w, const void* b,
                                const void* z, const float* mean, const float* rstd, void* dx,
                                float* dw, float* db, void* dz, float* ws, int64_t rows, int D,
                                bool rms, int dtype, int w_dtype, hipStream_t st);
// rows of partial sums of dw (and as many of db) that launch_norm_backward writes
int norm_backward_parts(int64_t rows);

// Chunk-wise backward pass; ws holds backward_slots() * Hv tiles of
// backward_tile_bytes().  cu (nullable): nseq + 1 token offsets on the device,
// then L is the number of all tokens, else of each sequence's.
int64_t backward_slots(int nseq, int L, bool packed);
int64_t backward_tile_bytes(int dk, int dv);
// workgroups (of 512 work items) of the walks of packed sequences of bf16: of both kinds,
// in both directions, of nseq * Hv heads rounded up to eights
constexpr int64_t packed_walk_groups(int nseq, int Hv, int dv) {
  return ((int64_t)nseq * Hv + 7) / 8 * 8 * 2 * (dv / 16 + dv / 64);
}
hipError_t launch_backward(const void* Q, const void* K, const void* V, const float* beta,
                           const float* g, const void* dO, const float* S0, const float* dSf,
                           void* dQ, void* dK, void* dV, float* dbeta, float* dg, float* dS0,
                           float* ws, const int* cu, int nseq, int L, int Hk, int Hv, int dk,
                           int dv, int C, float scale, int dtype, hipStream_t st);

}  // namespace gdn
