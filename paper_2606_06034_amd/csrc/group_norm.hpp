// group_norm.hpp -- host-side launchers of group norm, channels last (internal;
// arguments validated by api_linear.cpp).
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

namespace gdn {

struct GroupArgs {
  const void *dy, *x, *w, *b, *z;
  const float *mean_in, *rstd_in;
  void *out, *dz;
  float *mean, *rstd, *dw, *db, *ws;
  int64_t N;
  int S, G, Cg, C;
  float eps;
  bool act, wbf;
  // set by the launchers
  int tpi, gw, nw;      // groups in registers
  int sparts, cblocks, nrows;  // groups read twice
};

hipError_t launch_group_forward(const GroupArgs& a, int dtype, hipStream_t st);
hipError_t launch_group_backward(const GroupArgs& a, int dtype, hipStream_t st);
// workgroups of the largest launch over groups that are read twice (else 0)
int64_t group_forward_blocks(int64_t N, int S, int G, int Cg, int dtype);
int64_t group_backward_blocks(int64_t N, int S, int G, int Cg, int dtype);
// floats of workspace (sums: with dw or db)
int64_t group_forward_workspace(int64_t N, int S, int G, int Cg, int dtype);
int64_t group_backward_workspace(int64_t N, int S, int G, int Cg, int dtype, bool sums = true);

}  // namespace gdn
