// The gated feed-forward block of subgraphs of few rows (gated_ff_sets.cu).
#pragma once

#include "internal.cuh"
#include "mask.cuh"

namespace ff {

struct SetArgs {
  const float *x, *dy;
  int64_t x_ld, dy_ld;
  const float *wg, *wu, *wd;
  float *h, *dg, *du;                  // work area, [rows x H]
  float *dwg, *dwu, *dwd;              // or nullptr
  float* out;                          // y or dx
  int64_t out_ld;
  int32_t F, H, F_out, act, masked;
  philox::Mask mask;
  // filled in by the launch
  const int32_t* part_ptr;
  int32_t h_blocks, out_blocks;        // blocks of 32 columns of h, and of y or dx
};

// Whether these kernels run.
bool few_rows_per_set(const gnnco_handle* h, const gnnco_gated_ff_desc* d);
int32_t launch_sets(gnnco_handle* h, SetArgs A, int64_t sets, bool backward, cudaStream_t st);

}  // namespace ff
