// What the parts of the orthogonalised update share (muon.cu: entry points; muon_small.cu: a warp per matrix; muon_tc.cu: matrices
// that stay on chip; muon_tiles.cu: larger ones).
#pragma once

#include "internal.cuh"

struct NsJob {
  const void* G;              // gradient (or the matrix to orthogonalise), [sets x r x c]
  float *m, *W;               // momentum and weights, or NULL: write the iterate to O
  void* O;
  const uint8_t* active;
  int64_t sets;
  int32_t r, c, k, n;         // X is k x n, k <= n
  int32_t g_bf16, o_bf16, transpose, nesterov, steps, vec4, prefetch;
  float mu, keep, step, eps;  // W = W * keep - step * X
  float a, b, cc;             // the polynomial's coefficients
  float p_scale;              // power of two that P = a I + b A + c A^2 is held at in float16
  void* scratch;
  int32_t* status;
};

// u * lift * f = u * scale / (|u| + eps), |u|^2 = norm2.  Where |u| + eps is so small that the factor would leave float32's range (and
// make 0 * inf of a zero gradient), u is lifted by a power of two first; everywhere else lift is 1.
struct NsFactor { float lift, f; };
__device__ __forceinline__ NsFactor ns_factor(double norm2, float eps, float scale) {
  const double q = sqrt(norm2) + (double)eps;
  const float lift = q < 1e-20 ? 0x1p96f : 1.0f;
  return {lift, (float)((double)scale / (q * (double)lift))};
}

// ---- muon_small.cu: short side up to 16, on the FMA units
bool ns_small_supported(int32_t k, int32_t n);
int32_t launch_ns_small(gnnco_handle* h, const NsJob& job, cudaStream_t st);

// ---- muon_tc.cu: whole iterations on chip for k, n <= 256
bool ns_on_chip_supported(const gnnco_handle* h, int32_t k, int32_t n);
size_t ns_on_chip_scratch_bytes(const gnnco_handle* h, int64_t sets, int32_t k, int32_t n);
int32_t launch_ns_on_chip(gnnco_handle* h, const NsJob& job, cudaStream_t st);

// ---- muon_tiles.cu: one tiled launch per product, for any size
bool ns_tiles_supported(int32_t k, int32_t n);
size_t ns_tiles_workspace_bytes(int64_t sets, int32_t k, int32_t n);
int32_t launch_ns_tiles(gnnco_handle* h, const NsJob& job, void* ws, cudaStream_t st);
