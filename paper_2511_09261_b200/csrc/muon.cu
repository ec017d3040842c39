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

size_t workspace_bytes(const gnnco_handle* h, int64_t sets, int32_t r, int32_t c) {
  const int32_t k = r < c ? r : c, n = r < c ? c : r;
  if (ns_small_supported(k, n)) return 0;
  return align_up(ns_on_chip_supported(h, k, n) ? ns_on_chip_scratch_bytes(h, sets, k, n) : ns_tiles_workspace_bytes(sets, k, n));
}

bool valid_sizes(int64_t sets, int32_t r, int32_t c) {
  return sets >= 1 && sets < ((int64_t)1 << 31) && r >= 1 && c >= 1 && (int64_t)r * c < ((int64_t)1 << 31) &&
         ns_tiles_supported(r < c ? r : c, r < c ? c : r);
}

// The singular values start in [0, 1] and go through s -> s (a + b s^2 + c s^4) in every step.  The largest magnitude that the
// values in [0, top] reach is taken step by step at the ends and the stationary points (roots of a + 3 b u + 5 c u^2, u = s^2);
// a coefficient set that leads past 2 is refused: 2 bounds every stored value.  *p_max: the largest |a + b u + c u^2| met.
bool coefficients_bounded(double a, double b, double c, int steps, double* p_max) {
  double top = 1.0;
  *p_max = 0.0;
  auto poly = [&](double u) { return a + u * (b + u * c); };
  double root[2] = {-1.0, -1.0};                           // of 5 c u^2 + 3 b u + a; the form that does not cancel where c is tiny
  const double disc = 9.0 * b * b - 20.0 * a * c;
  if (disc >= 0.0) {
    const double q = -0.5 * (3.0 * b + copysign(sqrt(disc), b));
    if (c != 0.0) root[0] = q / (5.0 * c);
    if (q != 0.0) root[1] = a / q;
  }
  for (int t = 0; t < steps; ++t) {
    const double u_top = top * top;
    double reach = fabs(top * poly(u_top));
    for (double u : root)
      if (u > 0.0 && u < u_top) reach = fmax(reach, fabs(sqrt(u) * poly(u)));
    const double vertex = c != 0.0 ? -b / (2.0 * c) : -1.0;
    double p = fmax(fabs(a), fabs(poly(u_top)));
    if (vertex > 0.0 && vertex < u_top) p = fmax(p, fabs(poly(vertex)));
    if (!(reach <= 2.0) || !(p <= 1e30)) return false;
    *p_max = fmax(*p_max, p);
    top = fmax(top, reach);
  }
  return true;
}

struct NsParams { int steps; float a, b, c, eps; float p_scale; };

template <typename TG, typename TO>
int32_t run_ns(gnnco_handle* h, int64_t sets, int32_t r, int32_t c, const TG* G, float* m, float* W, TO* O, float mu, int nesterov,
               float keep, float step, const uint8_t* active, const NsParams& P, void* ws, cudaStream_t st) {
  const bool tr = r > c;
  const int32_t k = tr ? c : r, n = tr ? r : c, count = r * c;
  NsJob J = {};
  J.G = G; J.m = m; J.W = W; J.O = O; J.active = active; J.sets = sets;
  J.r = r; J.c = c; J.k = k; J.n = n;
  J.g_bf16 = sizeof(TG) == 2; J.o_bf16 = sizeof(TO) == 2; J.transpose = tr; J.nesterov = nesterov; J.steps = P.steps;
  J.vec4 = !tr && c % 4 == 0 && sizeof(TG) == 4 && vec_ok(G, c, 4, 4) && (!m || vec_ok(m, c, 4, 4)) &&
           (W ? vec_ok(W, c, 4, 4) : vec_ok(O, c, (int)sizeof(TO), 4));
  // prefetches move whole 16-byte lines of matrices that start on one
  J.prefetch = sizeof(TG) == 4 && count % 4 == 0 && !((uintptr_t)G & 15) && !((uintptr_t)m & 15) && !((uintptr_t)W & 15);
  J.mu = mu; J.keep = keep; J.step = step; J.eps = P.eps; J.a = P.a; J.b = P.b; J.cc = P.c; J.p_scale = P.p_scale;
  J.scratch = ws; J.status = h->status;
  if (ns_small_supported(k, n)) return launch_ns_small(h, J, st);
  return ns_on_chip_supported(h, k, n) ? launch_ns_on_chip(h, J, st) : launch_ns_tiles(h, J, ws, st);
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
  *bytes = workspace_bytes(h, sets, rows, cols);
  return GNNCO_OK;
}

extern "C" int32_t gnnco_muon_update(gnnco_handle* h, int64_t sets, int32_t rows, int32_t cols, float* W, float* m, const float* dW,
                                     const gnnco_muon_params* p, void* ws, size_t ws_bytes, void* stream) {
  if (!h || !W || !m || !dW || !p || ((uintptr_t)ws & 255) || !valid_sizes(sets, rows, cols)) return GNNCO_INVALID_ARGUMENT;
  NsParams P{p->steps, p->a, p->b, p->c, p->eps, 1.0f};
  const int32_t rc = check_params(P);
  if (rc != GNNCO_OK) return rc;
  const size_t need = workspace_bytes(h, sets, rows, cols);
  if (ws_bytes < need) return GNNCO_WORKSPACE_TOO_SMALL;
  if (need > 0 && !ws) return GNNCO_INVALID_ARGUMENT;
  cudaStream_t st = static_cast<cudaStream_t>(stream);
  ProfScope prof_(h, K_MUON, st);
  weights_written(h, W, (size_t)sets * rows * cols * sizeof(float));
  const float step = p->lr * sqrtf(cols > rows ? (float)cols / (float)rows : 1.0f);
  return run_ns<float, float>(h, sets, rows, cols, dW, m, W, nullptr, p->momentum, p->nesterov, 1.0f - p->lr * p->weight_decay,
                              step, p->active, P, ws, st);
}

extern "C" int32_t gnnco_orthogonalise(gnnco_handle* h, int32_t in_dtype, int32_t out_dtype, int64_t sets, int32_t rows, int32_t cols,
                                       const void* G, void* O, const gnnco_muon_params* p, void* ws, size_t ws_bytes,
                                       void* stream) {
  if (!h || !G || !O || !p || ((uintptr_t)ws & 255) || !valid_sizes(sets, rows, cols)) return GNNCO_INVALID_ARGUMENT;
  if ((in_dtype != GNNCO_F32 && in_dtype != GNNCO_BF16) || (out_dtype != GNNCO_F32 && out_dtype != GNNCO_BF16))
    return GNNCO_UNSUPPORTED;
  NsParams P{p->steps, p->a, p->b, p->c, p->eps, 1.0f};
  const int32_t rc = check_params(P);
  if (rc != GNNCO_OK) return rc;
  const size_t need = workspace_bytes(h, sets, rows, cols);
  if (ws_bytes < need) return GNNCO_WORKSPACE_TOO_SMALL;
  if (need > 0 && !ws) return GNNCO_INVALID_ARGUMENT;
  cudaStream_t st = static_cast<cudaStream_t>(stream);
  ProfScope prof_(h, K_MUON, st);
  weights_written(h, O, (size_t)sets * rows * cols * (out_dtype == GNNCO_F32 ? sizeof(float) : 2));
  typedef __nv_bfloat16 B;
#define GNNCO_ORTHO(TG, TO) \
  return run_ns<TG, TO>(h, sets, rows, cols, (const TG*)G, nullptr, nullptr, (TO*)O, 0.0f, 0, 0.0f, 0.0f, p->active, P, ws, st)
  if (in_dtype == GNNCO_F32 && out_dtype == GNNCO_F32) GNNCO_ORTHO(float, float);
  if (in_dtype == GNNCO_F32) GNNCO_ORTHO(float, B);
  if (out_dtype == GNNCO_F32) GNNCO_ORTHO(B, float);
  GNNCO_ORTHO(B, B);
#undef GNNCO_ORTHO
}
