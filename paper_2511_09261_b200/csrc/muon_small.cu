// Newton-Schulz iterations of matrices whose short side is at most 16 (the output layer's d x 1 weights among them), on the FMA
// units: one warp per matrix, which stays in the warp's shared memory from gradient to updated weight.  A tensor-core tile
// has 128 rows, of which such a matrix fills an eighth at most, and its kernel's chain of phases takes 15 us and more per
// matrix however small that is; here the work is what the matrix needs, in float32.
//
//   A = X X^T    a lane owns pairs (i, l), l <= i, and walks the columns (rows are padded to an odd stride: no bank conflicts)
//   P            a lane owns entries of a I + b A + c A A
//   X' = P X     a lane owns columns: the column in registers, P broadcast from shared memory
#include <math.h>

#include "muon_internal.cuh"
#include "vec_io.cuh"

namespace {

constexpr int kMaxK = 16, kMaxN = 256, kWarps = 4;

__device__ __forceinline__ float load_g(const NsJob& J, int64_t at) {
  return J.g_bf16 ? __bfloat162float(static_cast<const __nv_bfloat16*>(J.G)[at]) : __ldcs(static_cast<const float*>(J.G) + at);
}

template <int K>                                           // short side rounded up: 1, 2, 4, 8, 16
__global__ void __launch_bounds__(32 * kWarps) ns_small(const NsJob J) {
  extern __shared__ float sm[];
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  const int k = J.k, n = J.n, stride = n | 1;
  float* const X = sm + warp * (K * stride + 2 * K * K);   // [K][stride]
  float* const A = X + K * stride;                         // [K][K]
  float* const P = A + K * K;                              // [K][K]
  // the pairs (i, l), l <= i, that this lane sums
  constexpr int kPairs = K * (K + 1) / 2, kMine = (kPairs + 31) / 32;
  int pair_i[kMine], pair_l[kMine];
#pragma unroll
  for (int t = 0; t < kMine; ++t) {
    int q = lane + 32 * t, i = 0;
    while (q > i) {
      ++i;
      q -= i;
    }
    pair_i[t] = i;
    pair_l[t] = q;
  }
  for (int64_t s = (int64_t)blockIdx.x * kWarps + warp; s < J.sets; s += (int64_t)gridDim.x * kWarps) {
    if (J.active && !J.active[s]) continue;
    const int64_t base = s * (int64_t)J.r * J.c;
    const int count = J.r * J.c;
    // element q of the matrix is X[i][j]; lanes along the matrix' own order
    auto place = [&](int q, int& i, int& j) {
      const int a = q / J.c, b = q - a * J.c;
      i = J.transpose ? b : a;
      j = J.transpose ? a : b;
    };
    double sum = 0.0;
    for (int q0 = 0; q0 < count; q0 += 128) {
      float g[4], mv[4];
#pragma unroll
      for (int u = 0; u < 4; ++u) {
        const int q = q0 + 32 * u + lane;
        g[u] = q < count ? load_g(J, base + q) : 0.0f;
        mv[u] = q < count && J.m ? __ldcs(J.m + base + q) : 0.0f;
      }
#pragma unroll
      for (int u = 0; u < 4; ++u) {
        const int q = q0 + 32 * u + lane;
        if (q >= count) continue;
        if (J.m) {
          const float v = J.mu * mv[u] + g[u];
          __stcs(J.m + base + q, v);
          g[u] = J.nesterov ? g[u] + J.mu * v : v;
        }
        int i, j;
        place(q, i, j);
        X[i * stride + j] = g[u];
        sum += (double)g[u] * (double)g[u];
      }
    }
#pragma unroll
    for (int d = 16; d > 0; d >>= 1) sum += __shfl_xor_sync(0xffffffffu, sum, d);
    const NsFactor by = ns_factor(sum, J.eps, 1.0f);
    __syncwarp();
    for (int j = lane; j < n; j += 32)
#pragma unroll
      for (int i = 0; i < K; ++i) X[i * stride + j] = i < k ? X[i * stride + j] * by.lift * by.f : 0.0f;
    __syncwarp();
    for (int step = 0; step < J.steps; ++step) {
#pragma unroll
      for (int p = 0; p < kMine; ++p) {
        if (lane + 32 * p >= kPairs) continue;
        const int i = pair_i[p], l = pair_l[p];
        const float *a = X + i * stride, *b = X + l * stride;
        float t[4] = {0.0f, 0.0f, 0.0f, 0.0f};
        int j = 0;
        for (; j + 4 <= n; j += 4)
#pragma unroll
          for (int u = 0; u < 4; ++u) t[u] = fmaf(a[j + u], b[j + u], t[u]);
        for (; j < n; ++j) t[0] = fmaf(a[j], b[j], t[0]);
        const float v = (t[0] + t[1]) + (t[2] + t[3]);
        A[i * K + l] = v;
        A[l * K + i] = v;
      }
      __syncwarp();
      for (int q = lane; q < K * K; q += 32) {
        const int i = q / K, l = q % K;
        float v = 0.0f;
#pragma unroll
        for (int u = 0; u < K; ++u) v = fmaf(A[i * K + u], A[u * K + l], v);
        P[q] = fmaf(J.cc, v, fmaf(J.b, A[q], i == l ? J.a : 0.0f));
      }
      __syncwarp();
      // two columns at a time, so that an entry of P is read once for both
      for (int j = lane; j < n; j += 64) {
        const int j2 = j + 32 < n ? j + 32 : j;
        float x[K], z[K];
#pragma unroll
        for (int u = 0; u < K; ++u) {
          x[u] = X[u * stride + j];
          z[u] = X[u * stride + j2];
        }
#pragma unroll
        for (int i = 0; i < K; ++i) {
          float y0 = 0.0f, y1 = 0.0f;
#pragma unroll
          for (int u = 0; u < K; ++u) {
            const float p = P[i * K + u];
            y0 = fmaf(p, x[u], y0);
            y1 = fmaf(p, z[u], y1);
          }
          X[i * stride + j] = y0;
          X[i * stride + j2] = y1;
        }
      }
      __syncwarp();
    }
    for (int q0 = 0; q0 < count; q0 += 128) {
      float w[4];
#pragma unroll
      for (int u = 0; u < 4; ++u) w[u] = J.W && q0 + 32 * u + lane < count ? __ldcs(J.W + base + q0 + 32 * u + lane) : 0.0f;
#pragma unroll
      for (int u = 0; u < 4; ++u) {
        const int q = q0 + 32 * u + lane;
        if (q >= count) continue;
        int i, j;
        place(q, i, j);
        const float x = X[i * stride + j];
        if (J.W) __stcs(J.W + base + q, w[u] * J.keep - J.step * x);
        else if (J.o_bf16) static_cast<__nv_bfloat16*>(J.O)[base + q] = __float2bfloat16_rn(x);
        else __stcs(static_cast<float*>(J.O) + base + q, x);
      }
    }
    __syncwarp();
  }
}

template <int K>
int32_t launch(gnnco_handle* h, const NsJob& J, cudaStream_t st) {
  const size_t bytes = kWarps * ((size_t)K * (J.n | 1) + 2 * K * K) * sizeof(float);
  static std::atomic<int> allowed{0};
  constexpr size_t most = kWarps * ((size_t)K * (kMaxN | 1) + 2 * K * K) * sizeof(float);
  const int32_t rc = allow_shared_memory(ns_small<K>, most, h->device, allowed);
  if (rc != GNNCO_OK) return rc;
  const int64_t need = (J.sets + kWarps - 1) / kWarps, blocks = (int64_t)h->sm_count * 16;
  ns_small<K><<<(unsigned)(need < blocks ? need : blocks), 32 * kWarps, bytes, st>>>(J);
  h->launches += 1;
  GNNCO_LAUNCH_CHECK();
  return GNNCO_OK;
}

}  // namespace

// 4,096 sets take 48 us at 256 x 1, 156 at 256 x 8 and 474 at 16 x 256 here, 1,203, 1,298 and 720 us on the tensor cores.  (Two sets of
// 8 x 256 take 50 us here and 27 there; the choice does not go by the number of sets, so that neither do the bits.)
bool ns_small_supported(int32_t k, int32_t n) { return k <= kMaxK && n <= kMaxN; }

int32_t launch_ns_small(gnnco_handle* h, const NsJob& job, cudaStream_t st) {
  if (job.k <= 1) return launch<1>(h, job, st);
  if (job.k <= 2) return launch<2>(h, job, st);
  if (job.k <= 4) return launch<4>(h, job, st);
  if (job.k <= 8) return launch<8>(h, job, st);
  return launch<16>(h, job, st);
}
