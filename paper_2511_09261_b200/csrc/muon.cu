// Weight updates orthogonalised by Newton-Schulz products, for a batch of matrices (one weight per subgraph, or one shared
// weight):
//
//   m  = mu m + g,   u = g + mu m (Nesterov) or m
//   X  = u / (|u|_F + eps), transposed where rows > cols, so that X is k x n with k <= n
//   `steps` times:   A = X X^T,   X = (a I + b A + c A A) X
//   W  = W (1 - lr wd) - lr sqrt(max(1, cols / rows)) X
//
// W is [d_in, d_out] (a layer computes H W), so cols / rows is fan-out over fan-in.  The iteration moves every singular
// value of u towards 1 and leaves the singular vectors alone.
#include <math.h>

#include "muon_internal.cuh"
#include "vec_io.cuh"

namespace {

constexpr int kPartials = 64;                              // partial sums of squares per matrix, at most

// ---- m, u and the sum of squares: grid (blocks, sets)
template <typename T>
__global__ void __launch_bounds__(256) muon_begin(const T* __restrict__ G, float* __restrict__ m, float* __restrict__ X,
                                                  double* __restrict__ partial, int32_t r, int32_t c, bool transpose, float mu,
                                                  int nesterov, const uint8_t* __restrict__ active, int64_t set0) {
  const int64_t s = blockIdx.y, base = (set0 + s) * (int64_t)r * c, xbase = s * (int64_t)r * c;
  if (active && !active[set0 + s]) return;
  const int32_t count = r * c;
  double sum = 0.0;
  for (int32_t q = blockIdx.x * 256 + threadIdx.x; q < count; q += gridDim.x * 256) {
    vio::Raw<T, 1> g1;
    g1.template load<true>(G + base + q);
    float u = g1.get(0);
    if (m) {
      const float mq = mu * m[base + q] + u;
      m[base + q] = mq;
      u = nesterov ? u + mu * mq : mq;
    }
    const int32_t i = q / c, j = q - i * c;
    X[xbase + (transpose ? (int64_t)j * r + i : (int64_t)q)] = u;
    sum += (double)u * (double)u;
  }
  __shared__ double w[8];
#pragma unroll
  for (int d = 16; d > 0; d >>= 1) sum += __shfl_xor_sync(0xffffffffu, sum, d);
  if ((threadIdx.x & 31) == 0) w[threadIdx.x >> 5] = sum;
  __syncthreads();
  if (threadIdx.x == 0) {
    double t = 0.0;
    for (int i = 0; i < 8; ++i) t += w[i];
    partial[s * gridDim.x + blockIdx.x] = t;
  }
}

__global__ void __launch_bounds__(256) muon_scale(float* __restrict__ X, const double* __restrict__ partial, int parts, int32_t count,
                                                  float eps, const uint8_t* __restrict__ active, int64_t set0) {
  const int64_t s = blockIdx.y;
  if (active && !active[set0 + s]) return;
  double t = 0.0;
  for (int i = 0; i < parts; ++i) t += partial[s * parts + i];
  const float f = (float)(1.0 / (sqrt(t) + (double)eps));
  for (int32_t q = blockIdx.x * 256 + threadIdx.x; q < count; q += gridDim.x * 256) X[s * count + q] *= f;
}

// D = alpha A op(B) + beta C + gamma I, all row-major float32, op(B) = B^T when trans_b; grid (n / 64, m / 64, sets)
__global__ void __launch_bounds__(256) muon_product(const float* __restrict__ A, const float* __restrict__ B, const float* __restrict__ C,
                                                    float* __restrict__ D, int32_t M, int32_t N, int32_t K, bool trans_b,
                                                    float alpha, float beta, float gamma, const uint8_t* __restrict__ active,
                                                    int64_t set0) {
  const int64_t s = blockIdx.z;
  if (active && !active[set0 + s]) return;
  A += s * (int64_t)M * K;
  B += s * (int64_t)N * K;
  D += s * (int64_t)M * N;
  if (C) C += s * (int64_t)M * N;
  __shared__ float sa[16][65], sb[16][65];
  const int tx = threadIdx.x & 15, ty = threadIdx.x >> 4;
  const int i0 = blockIdx.y * 64, j0 = blockIdx.x * 64;
  float acc[4][4] = {};
  for (int k0 = 0; k0 < K; k0 += 16) {
    for (int q = threadIdx.x; q < 1024; q += 256) {
      const int i = q >> 4, k = q & 15;
      sa[k][i] = i0 + i < M && k0 + k < K ? A[(int64_t)(i0 + i) * K + k0 + k] : 0.0f;
      if (trans_b) {
        sb[k][i] = j0 + i < N && k0 + k < K ? B[(int64_t)(j0 + i) * K + k0 + k] : 0.0f;
      } else {
        const int kk = q >> 6, j = q & 63;
        sb[kk][j] = j0 + j < N && k0 + kk < K ? B[(int64_t)(k0 + kk) * N + j0 + j] : 0.0f;
      }
    }
    __syncthreads();
#pragma unroll
    for (int k = 0; k < 16; ++k) {
      float a[4], b[4];
#pragma unroll
      for (int u = 0; u < 4; ++u) {
        a[u] = sa[k][ty + 16 * u];
        b[u] = sb[k][tx + 16 * u];
      }
#pragma unroll
      for (int u = 0; u < 4; ++u)
#pragma unroll
        for (int v = 0; v < 4; ++v) acc[u][v] += a[u] * b[v];
    }
    __syncthreads();
  }
#pragma unroll
  for (int u = 0; u < 4; ++u)
#pragma unroll
    for (int v = 0; v < 4; ++v) {
      const int i = i0 + ty + 16 * u, j = j0 + tx + 16 * v;
      if (i < M && j < N) {
        float d = alpha * acc[u][v];
        if (C) d += beta * C[(int64_t)i * N + j];
        if (i == j) d += gamma;
        D[(int64_t)i * N + j] = d;
      }
    }
}

template <typename T>
__global__ void __launch_bounds__(256) muon_finish(const float* __restrict__ X, float* __restrict__ W, T* __restrict__ O, int32_t r,
                                                   int32_t c, bool transpose, float keep, float step,
                                                   const uint8_t* __restrict__ active, int64_t set0) {
  const int64_t s = blockIdx.y, base = (set0 + s) * (int64_t)r * c, xbase = s * (int64_t)r * c;
  if (active && !active[set0 + s]) return;
  const int32_t count = r * c;
  for (int32_t q = blockIdx.x * 256 + threadIdx.x; q < count; q += gridDim.x * 256) {
    const int32_t i = q / c, j = q - i * c;
    const float x = X[xbase + (transpose ? (int64_t)j * r + i : (int64_t)q)];
    if (W) {
      W[base + q] = W[base + q] * keep - step * x;
    } else {
      float f[1] = {x};
      vio::store_stream<T, 1>(O + base + q, f);
    }
  }
}

struct NsLayout {
  float *x0, *x1, *a, *p;
  double* partial;
  void* scratch;                                           // of the on-chip kernel, where that one runs
  bool on_chip;
  int64_t chunk;                                           // matrices worked on at a time
  size_t bytes;
};
NsLayout ns_layout(const gnnco_handle* h, void* ws, int64_t sets, int64_t r, int64_t c) {
  const int64_t k = r < c ? r : c, n = r < c ? c : r;
  NsLayout L = {};
  Carver cv(ws, 0);
  L.on_chip = ns_on_chip_supported(h, (int32_t)k, (int32_t)n);
  if (L.on_chip) {
    L.scratch = cv.take<char>(ns_on_chip_scratch_bytes(h, sets, (int32_t)k, (int32_t)n));
    L.bytes = cv.off;
    return L;
  }
  const int64_t each = (2 * r * c + 2 * k * k) * 4;
  L.chunk = ((int64_t)256 << 20) / each;
  if (L.chunk < 1) L.chunk = 1;
  if (L.chunk > sets) L.chunk = sets;
  if (L.chunk > 32768) L.chunk = 32768;
  L.x0 = cv.take<float>(L.chunk * r * c);
  L.x1 = cv.take<float>(L.chunk * r * c);
  L.a = cv.take<float>(L.chunk * k * k);
  L.p = cv.take<float>(L.chunk * k * k);
  L.partial = cv.take<double>(L.chunk * kPartials);
  L.bytes = cv.off;
  return L;
}

bool valid_sizes(int64_t sets, int32_t r, int32_t c) {
  return sets >= 1 && sets < ((int64_t)1 << 31) && r >= 1 && c >= 1 && (int64_t)r * c < ((int64_t)1 << 31);
}

// The iteration must stay bounded on [0, 1], where the singular values start; what it reaches there also bounds every
// intermediate value.  Sampled densely; a coefficient set whose values grow past 2 is refused.  *p_max: the largest
// |a + b s^2 + c s^4| over the values reached.
bool coefficients_bounded(float a, float b, float c, int steps, double* p_max) {
  double top = 1.0;
  for (int q = 0; q <= 4096; ++q) {
    double s = q / 4096.0;
    for (int t = 0; t < steps; ++t) {
      const double s2 = s * s;
      s = s * (a + s2 * (b + s2 * (double)c));
      if (!(fabs(s) <= 2.0)) return false;
      if (fabs(s) > top) top = fabs(s);
    }
  }
  *p_max = 0.0;
  for (int q = 0; q <= 4096; ++q) {
    const double s = top * q / 4096.0, s2 = s * s, p = fabs(a + s2 * (b + s2 * (double)c));
    if (p > *p_max) *p_max = p;
  }
  return true;
}

struct NsParams { int steps; float a, b, c, eps; float p_scale; };

template <typename TG, typename TO>
int32_t run_ns(gnnco_handle* h, int64_t sets, int32_t r, int32_t c, const TG* G, float* m, float* W, TO* O, float mu, int nesterov,
               float keep, float step, const uint8_t* active, const NsParams& P, const NsLayout& L, cudaStream_t st) {
  const bool tr = r > c;
  const int32_t k = tr ? c : r, n = tr ? r : c, count = r * c;
  if (L.on_chip) {
    NsJob J = {};
    J.G = G; J.m = m; J.W = W; J.O = O; J.active = active; J.sets = sets;
    J.r = r; J.c = c; J.k = k; J.n = n;
    J.g_bf16 = sizeof(TG) == 2; J.o_bf16 = sizeof(TO) == 2; J.transpose = tr; J.nesterov = nesterov; J.steps = P.steps;
    J.vec4 = !tr && c % 4 == 0 && sizeof(TG) == 4 && vec_ok(G, c, 4, 4) && (!m || vec_ok(m, c, 4, 4)) &&
             (W ? vec_ok(W, c, 4, 4) : vec_ok(O, c, (int)sizeof(TO), 4));
    // prefetches move whole 16-byte lines of matrices that start on one
    J.prefetch = sizeof(TG) == 4 && count % 4 == 0 && !((uintptr_t)G & 15) && !((uintptr_t)m & 15) && !((uintptr_t)W & 15);
    J.mu = mu; J.keep = keep; J.step = step; J.eps = P.eps; J.a = P.a; J.b = P.b; J.cc = P.c; J.p_scale = P.p_scale;
    J.scratch = L.scratch; J.status = h->status;
    return launch_ns_on_chip(h, J, st);
  }
  int parts = (count + 4095) / 4096;
  if (parts > kPartials) parts = kPartials;
  for (int64_t s0 = 0; s0 < sets; s0 += L.chunk) {
    const unsigned ns = (unsigned)(sets - s0 < L.chunk ? sets - s0 : L.chunk);
    float *x = L.x0, *y = L.x1;
    muon_begin<TG><<<dim3(parts, ns), 256, 0, st>>>(G, m, x, L.partial, r, c, tr, mu, nesterov, active, s0);
    muon_scale<<<dim3(parts, ns), 256, 0, st>>>(x, L.partial, parts, count, P.eps, active, s0);
    for (int t = 0; t < P.steps; ++t) {
      const unsigned kb = (k + 63) / 64, nb = (n + 63) / 64;
      muon_product<<<dim3(kb, kb, ns), 256, 0, st>>>(x, x, nullptr, L.a, k, k, n, true, 1.0f, 0.0f, 0.0f, active, s0);
      muon_product<<<dim3(kb, kb, ns), 256, 0, st>>>(L.a, L.a, L.a, L.p, k, k, k, true, P.c, P.b, P.a, active, s0);
      muon_product<<<dim3(nb, kb, ns), 256, 0, st>>>(L.p, x, nullptr, y, k, n, k, false, 1.0f, 0.0f, 0.0f, active, s0);
      float* q = x; x = y; y = q;
    }
    muon_finish<TO><<<dim3(parts, ns), 256, 0, st>>>(x, W, O, r, c, tr, keep, step, active, s0);
    h->launches += 3 + 3 * P.steps;
  }
  GNNCO_LAUNCH_CHECK();
  return GNNCO_OK;
}

int32_t check_params(NsParams& P) {
  if (P.steps < 1 || P.steps > 32 || !(P.eps > 0.0f)) return GNNCO_INVALID_ARGUMENT;
  double p_max = 0.0;
  if (!coefficients_bounded(P.a, P.b, P.c, P.steps, &p_max)) return GNNCO_INVALID_ARGUMENT;
  // entries of P stay below 2^15 in float16
  P.p_scale = 16384.0f;
  while (P.p_scale * p_max > 32768.0) P.p_scale *= 0.5f;
  return GNNCO_OK;
}

}  // namespace

extern "C" int32_t gnnco_muon_workspace_bytes(const gnnco_handle* h, int64_t sets, int32_t rows, int32_t cols, size_t* bytes) {
  if (!h || !bytes || !valid_sizes(sets, rows, cols)) return GNNCO_INVALID_ARGUMENT;
  *bytes = ns_layout(h, nullptr, sets, rows, cols).bytes;
  return GNNCO_OK;
}

extern "C" int32_t gnnco_muon_update(gnnco_handle* h, int64_t sets, int32_t rows, int32_t cols, float* W, float* m, const float* dW,
                                     const gnnco_muon_params* p, void* ws, size_t ws_bytes, void* stream) {
  if (!h || !W || !m || !dW || !p || !ws || ((uintptr_t)ws & 255) || !valid_sizes(sets, rows, cols)) return GNNCO_INVALID_ARGUMENT;
  NsParams P{p->steps, p->a, p->b, p->c, p->eps, 1.0f};
  const int32_t rc = check_params(P);
  if (rc != GNNCO_OK) return rc;
  const NsLayout L = ns_layout(h, ws, sets, rows, cols);
  if (ws_bytes < L.bytes) return GNNCO_WORKSPACE_TOO_SMALL;
  cudaStream_t st = static_cast<cudaStream_t>(stream);
  ProfScope prof_(h, K_MUON, st);
  // the bf16 copies of these weights that an earlier step left behind are stale from here on
  for (int l = 0; l < GNNCO_MAX_LAYERS; ++l)
    if (h->shadow_W[l] == W) h->shadow_fresh[l] = false;
  const float step = p->lr * sqrtf(cols > rows ? (float)cols / (float)rows : 1.0f);
  return run_ns<float, float>(h, sets, rows, cols, dW, m, W, nullptr, p->momentum, p->nesterov, 1.0f - p->lr * p->weight_decay,
                              step, p->active, P, L, st);
}

extern "C" int32_t gnnco_orthogonalise(gnnco_handle* h, int32_t in_dtype, int32_t out_dtype, int64_t sets, int32_t rows, int32_t cols,
                                       const void* G, void* O, const gnnco_muon_params* p, void* ws, size_t ws_bytes,
                                       void* stream) {
  if (!h || !G || !O || !p || !ws || ((uintptr_t)ws & 255) || !valid_sizes(sets, rows, cols)) return GNNCO_INVALID_ARGUMENT;
  if ((in_dtype != GNNCO_F32 && in_dtype != GNNCO_BF16) || (out_dtype != GNNCO_F32 && out_dtype != GNNCO_BF16))
    return GNNCO_UNSUPPORTED;
  NsParams P{p->steps, p->a, p->b, p->c, p->eps, 1.0f};
  const int32_t rc = check_params(P);
  if (rc != GNNCO_OK) return rc;
  const NsLayout L = ns_layout(h, ws, sets, rows, cols);
  if (ws_bytes < L.bytes) return GNNCO_WORKSPACE_TOO_SMALL;
  cudaStream_t st = static_cast<cudaStream_t>(stream);
  ProfScope prof_(h, K_MUON, st);
  typedef __nv_bfloat16 B;
#define GNNCO_ORTHO(TG, TO) \
  return run_ns<TG, TO>(h, sets, rows, cols, (const TG*)G, nullptr, nullptr, (TO*)O, 0.0f, 0, 0.0f, 0.0f, p->active, P, L, st)
  if (in_dtype == GNNCO_F32 && out_dtype == GNNCO_F32) GNNCO_ORTHO(float, float);
  if (in_dtype == GNNCO_F32) GNNCO_ORTHO(float, B);
  if (out_dtype == GNNCO_F32) GNNCO_ORTHO(B, float);
  GNNCO_ORTHO(B, B);
#undef GNNCO_ORTHO
}
