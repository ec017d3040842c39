// Norms before and after a block of the network, fused with the block's gate and residual scale:
//
//   r(v) = 1 / sqrt(mean_f v_f^2 + eps)
//   x'   = x + s * g .* (y * r(y)) .* w_post         norm after the block (output y), gate g, residual scale s
//   h    = (x' * r(x')) .* w_pre                     norm before the next block
//
// and the gradient of both, with xh = x' r(x'), yh = y r(y), a = dh .* w_pre, b = s g .* w_post .* D:
//
//   D    = dx' + r(x') (a - xh mean(a .* xh)),  dx = D,   dy = r(y) (b - yh mean(b .* yh))
//   dw_pre = sum dh .* xh,   dw_post = sum s g .* D .* yh,   dg = s D .* w_post .* yh (summed over rows if g is shared)
//
// One pass over memory each way: a row stays in the registers of its team of lanes, both means are taken there, and the
// row statistics are recomputed in the backward pass (the rows are read anyway).  Both kernels are bound by HBM.
// Sums over rows are kept per lane in float32, joined over the block's teams in shared memory and over blocks by a
// second kernel, always in the same order: no atomics.
#include "internal.cuh"
#include "vec_io.cuh"

namespace {

template <int TEAM>
struct TeamSum {
  static __device__ __forceinline__ float one(float a, float2* buf) {
    if constexpr (TEAM <= 32) {
#pragma unroll
      for (int d = TEAM / 2; d > 0; d >>= 1) a += __shfl_xor_sync(0xffffffffu, a, d);
      return a;
    } else {
      return both(a, 0.0f, buf).x;
    }
  }
  // sum of a and of b over the team, returned to every lane
  static __device__ __forceinline__ float2 both(float a, float b, float2* buf) {
    if constexpr (TEAM <= 32) {
#pragma unroll
      for (int d = TEAM / 2; d > 0; d >>= 1) {
        a += __shfl_xor_sync(0xffffffffu, a, d);
        b += __shfl_xor_sync(0xffffffffu, b, d);
      }
      return make_float2(a, b);
    } else {
#pragma unroll
      for (int d = 16; d > 0; d >>= 1) {
        a += __shfl_xor_sync(0xffffffffu, a, d);
        b += __shfl_xor_sync(0xffffffffu, b, d);
      }
      __syncthreads();                                     // buf may still be read from the sum before
      if ((threadIdx.x & 31) == 0) buf[threadIdx.x >> 5] = make_float2(a, b);
      __syncthreads();
      float2 t = make_float2(0.0f, 0.0f);
#pragma unroll
      for (int w = 0; w < TEAM / 32; ++w) {
        t.x += buf[w].x;
        t.y += buf[w].y;
      }
      return t;
    }
  }
};

struct NormArgs {
  const void *x, *y, *gate;
  const float *w_pre, *w_post;
  const void *dx_out, *dh;
  void *x_out, *h_out, *dx, *dy, *dgate;
  float* partial;                                          // [blocks][2][F]: sum dh .* xh, and sum (g s) D .* yh
  int64_t x_ld, y_ld, gate_ld, dx_out_ld, dh_ld, x_out_ld, h_out_ld, dx_ld, dy_ld, dgate_ld;
  int64_t rows;
  int32_t F;
  float scale, eps, inv_F;
};

// what the gate is
constexpr int kGateNone = 0, kGateVector = 1, kGateRows = 2;

// A lane's share of a vector of F float32 weights: 1 where there is none, times f.
template <int VEC, int TEAM, int K>
__device__ __forceinline__ void lane_weights(vio::Vec<VEC> (&w)[K], const float* p, int F, int tl, float f) {
#pragma unroll
  for (int k = 0; k < K; ++k)
#pragma unroll
    for (int e = 0; e < VEC; ++e) {
      const int col = (k * TEAM + tl) * VEC + e;
      w[k].v[e] = col < F ? f * (p ? __ldg(p + col) : 1.0f) : 0.0f;
    }
}
// s w_post, times g where the gate is shared
template <int VEC, int TEAM, int K>
__device__ __forceinline__ void post_weights(vio::Vec<VEC> (&c)[K], const NormArgs& A, int gate_kind, int tl) {
  lane_weights<VEC, TEAM, K>(c, A.w_post, A.F, tl, A.scale);
  if (gate_kind != kGateVector) return;
#pragma unroll
  for (int k = 0; k < K; ++k)
#pragma unroll
    for (int e = 0; e < VEC; ++e) {
      const int col = (k * TEAM + tl) * VEC + e;
      if (col < A.F) c[k].v[e] *= __ldg((const float*)A.gate + col);
    }
}
__device__ __forceinline__ float inverse_rms(float sum_of_squares, const NormArgs& A) {
  // 2 units in the last place at most.  (The correctly rounded root takes dx and dy of 100,003 x 99 from 4.8e-8 and 7.9e-8 of their norms to
  // 4.5e-8 and 7.4e-8, and the backward pass of it from 75 to 85 us, of 2.5M x 256 bf16 from 1,386 to 1,578 us.)
  return rsqrtf(sum_of_squares * A.inv_F + A.eps);
}

// Teams of TEAM lanes, K vectors of VEC elements per lane; blocks go through the rows grid-stride, weights stay in
// registers.  2.5M x 256 bf16: 895 us (5.7 TB/s); 911 with the registers of four blocks per SM, 970 with five; two rows of a team in
// flight at a time changed nothing.
template <typename T, int VEC, int TEAM, int K>
__global__ void __launch_bounds__(TEAM > 256 ? TEAM : 256)
norm_forward(const NormArgs A, const int gate_kind) {
  using V = vio::Vec<VEC>;
  constexpr int THREADS = TEAM > 256 ? TEAM : 256, TEAMS = THREADS / TEAM;
  __shared__ float2 buf[TEAM > 32 ? TEAM / 32 : 1];
  const int tl = threadIdx.x % TEAM, team = threadIdx.x / TEAM;
  V c_post[K], w_pre[K];
  lane_weights<VEC, TEAM, K>(w_pre, A.w_pre, A.F, tl, 1.0f);
  post_weights<VEC, TEAM, K>(c_post, A, gate_kind, tl);
  // whole blocks stay in the loop together (the sums name all lanes)
  for (int64_t lead = (int64_t)blockIdx.x * TEAMS; lead < A.rows; lead += (int64_t)gridDim.x * TEAMS) {
    const int64_t row = lead + team;
    vio::Raw<T, VEC> xr[K], yr[K], gr[K];
#pragma unroll
    for (int k = 0; k < K; ++k) {
      const int col = (k * TEAM + tl) * VEC;
      const bool in = row < A.rows && col < A.F;
      if (in) xr[k].template load<true>((const T*)A.x + row * A.x_ld + col);
      else xr[k].zero();
      if (in && A.y) yr[k].template load<true>((const T*)A.y + row * A.y_ld + col);
      else yr[k].zero();
      gr[k].zero();
      if (gate_kind == kGateRows && in) gr[k].template load<true>((const T*)A.gate + row * A.gate_ld + col);
    }
    V xo[K], sq(0.0f);
    if (A.y) {
#pragma unroll
      for (int k = 0; k < K; ++k) sq = vio::fma(V(yr[k]), V(yr[k]), sq);
      const float f = inverse_rms(TeamSum<TEAM>::one(sq.sum(), buf), A);
      sq = V(0.0f);
#pragma unroll
      for (int k = 0; k < K; ++k) {
        const int col = (k * TEAM + tl) * VEC;
        V c = vio::mul(c_post[k], f);
        if (gate_kind == kGateRows) c = vio::mul(c, V(gr[k]));
        xo[k] = vio::fma(c, V(yr[k]), V(xr[k]));
        sq = vio::fma(xo[k], xo[k], sq);
        if (row < A.rows && col < A.F) vio::store_stream<T, VEC>((T*)A.x_out + row * A.x_out_ld + col, xo[k].v);
      }
    } else {
#pragma unroll
      for (int k = 0; k < K; ++k) {
        xo[k] = V(xr[k]);
        sq = vio::fma(xo[k], xo[k], sq);
      }
    }
    if (!A.h_out) continue;
    const float rx = inverse_rms(TeamSum<TEAM>::one(sq.sum(), buf), A);
#pragma unroll
    for (int k = 0; k < K; ++k) {
      const int col = (k * TEAM + tl) * VEC;
      if (row >= A.rows || col >= A.F) continue;
      vio::store_stream<T, VEC>((T*)A.h_out + row * A.h_out_ld + col, vio::mul(xo[k], vio::mul(w_pre[k], rx)).v);
    }
  }
}

// Three blocks per SM where a lane holds at most eight elements: 2.5M x 256 bf16 takes 1,426 us so (5.4 TB/s), 1,548 with two and 1,688
// with four, whose registers spill.
template <typename T, int VEC, int TEAM, int K>
__global__ void __launch_bounds__(TEAM > 256 ? TEAM : 256, TEAM > 256 ? 1 : K * VEC <= 8 ? 3 : 1)
norm_backward(const NormArgs A, const int gate_kind) {
  using V = vio::Vec<VEC>;
  constexpr int THREADS = TEAM > 256 ? TEAM : 256, TEAMS = THREADS / TEAM;
  __shared__ float2 buf[TEAM > 32 ? TEAM / 32 : 1];
  extern __shared__ float join[];                          // [TEAMS][TEAM * K * VEC], one quantity at a time
  const int tl = threadIdx.x % TEAM, team = threadIdx.x / TEAM;
  V s_pre[K], s_post[K], c_post[K], w_pre[K];
#pragma unroll
  for (int k = 0; k < K; ++k) s_pre[k] = s_post[k] = V(0.0f);
  lane_weights<VEC, TEAM, K>(w_pre, A.w_pre, A.F, tl, 1.0f);
  post_weights<VEC, TEAM, K>(c_post, A, gate_kind, tl);
  for (int64_t lead = (int64_t)blockIdx.x * TEAMS; lead < A.rows; lead += (int64_t)gridDim.x * TEAMS) {
    const int64_t row = lead + team;
    vio::Raw<T, VEC> xr[K], yr[K], dr[K], hr[K], gr[K];
#pragma unroll
    for (int k = 0; k < K; ++k) {
      const int col = (k * TEAM + tl) * VEC;
      const bool in = row < A.rows && col < A.F;
      if (in && A.dh) {
        xr[k].template load<true>((const T*)A.x + row * A.x_ld + col);
        hr[k].template load<true>((const T*)A.dh + row * A.dh_ld + col);
      } else {
        xr[k].zero();
        hr[k].zero();
      }
      if (in && A.y) yr[k].template load<true>((const T*)A.y + row * A.y_ld + col);
      else yr[k].zero();
      if (in && A.dx_out) dr[k].template load<true>((const T*)A.dx_out + row * A.dx_out_ld + col);
      else dr[k].zero();
      gr[k].zero();
      if (gate_kind == kGateRows && in) gr[k].template load<true>((const T*)A.gate + row * A.gate_ld + col);
    }
    // mean over features of x'^2 and of a .* x'
    V sx(0.0f), sa(0.0f);
#pragma unroll
    for (int k = 0; k < K; ++k) {
      const V x(xr[k]);
      sx = vio::fma(x, x, sx);
      sa = vio::fma(vio::mul(V(hr[k]), w_pre[k]), x, sa);
    }
    float2 t = TeamSum<TEAM>::both(sx.sum(), sa.sum(), buf);
    const float rx = inverse_rms(t.x, A);
    const float cx = t.y * A.inv_F * rx * rx;               // mean(a .* xh) r(x'): times x' below
    V D[K], sy(0.0f), sb(0.0f);
#pragma unroll
    for (int k = 0; k < K; ++k) {
      const int col = (k * TEAM + tl) * VEC;
      const V x(xr[k]), h(hr[k]), y(yr[k]), xh = vio::mul(x, rx);
      s_pre[k] = vio::fma(h, xh, s_pre[k]);
      D[k] = vio::fma(vio::mul(h, w_pre[k]), rx, vio::fma(xh, -cx, V(dr[k])));
      V c = vio::mul(c_post[k], D[k]);
      if (gate_kind == kGateRows) c = vio::mul(c, V(gr[k]));
      sy = vio::fma(y, y, sy);
      sb = vio::fma(c, y, sb);
      if (row < A.rows && col < A.F) vio::store_stream<T, VEC>((T*)A.dx + row * A.dx_ld + col, D[k].v);
    }
    if (!A.y) continue;                                    // the same for all rows: no lane is left alone
    t = TeamSum<TEAM>::both(sy.sum(), sb.sum(), buf);
    const float ry = inverse_rms(t.x, A);
    const float cy = t.y * A.inv_F * ry * ry;
#pragma unroll
    for (int k = 0; k < K; ++k) {
      const int col = (k * TEAM + tl) * VEC;
      const bool in = row < A.rows && col < A.F;
      const V y(yr[k]), yh = vio::mul(y, ry), q = vio::mul(D[k], yh);   // q, times s: the shared factor of dg and dw_post
      V c = vio::mul(c_post[k], D[k]);
      if (gate_kind == kGateRows) {
        const V g(gr[k]);
        s_post[k] = vio::fma(g, q, s_post[k]);
        if (in && A.dgate) vio::store_stream<T, VEC>((T*)A.dgate + row * A.dgate_ld + col, vio::mul(c_post[k], q).v);
        c = vio::mul(c, g);
      } else {
        s_post[k] = vio::fma(D[k], yh, s_post[k]);
      }
      if (in) vio::store_stream<T, VEC>((T*)A.dy + row * A.dy_ld + col, vio::fma(c, ry, vio::mul(yh, -cy)).v);
    }
  }

  constexpr int W = TEAM * K * VEC;
#pragma unroll
  for (int which = 0; which < 2; ++which) {
    __syncthreads();
#pragma unroll
    for (int k = 0; k < K; ++k)
#pragma unroll
      for (int e = 0; e < VEC; ++e) join[team * W + (k * TEAM + tl) * VEC + e] = which == 0 ? s_pre[k].v[e] : s_post[k].v[e];
    __syncthreads();
    for (int f = threadIdx.x; f < A.F; f += THREADS) {
      float s = 0.0f;
#pragma unroll 4
      for (int q = 0; q < TEAMS; ++q) s += join[q * W + f];
      A.partial[((int64_t)blockIdx.x * 2 + which) * A.F + f] = which == 0 ? s : A.scale * s;
    }
  }
}

// Sums over the blocks' partial sums: a warp takes every 32nd block, four at a time, and the fours and the warps' sums are added as
// trees, always in the same order.  100,003 x 99 with a gate per row: dw_pre and dw_post are 1.6e-7 and 1.75e-7 of their norms off
// (one running sum each way: 1.9e-7 and 2.0e-7 in the same time; in float64: 1.3e-7 and 1.5e-7, 1.3 us more).
//   dw_pre = S0;  shared gate (or none): S1 = sum s D .* yh, dg = w_post S1, dw_post = g S1;  gate per row: dw_post = S1
__global__ void __launch_bounds__(1024) norm_weight_sums(const float* __restrict__ partial, int blocks, int32_t F,
                                                         const float* __restrict__ gate, const float* __restrict__ w_post,
                                                         float* dw_pre, float* dw_post, float* dgate) {
  __shared__ float s0[32][33], s1[32][33];
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  const int col = blockIdx.x * 32 + lane;
  float a = 0.0f, b = 0.0f;
  if (col < F)
    for (int q = warp; q < blocks; q += 128) {
      float va[4], vb[4];
#pragma unroll
      for (int u = 0; u < 4; ++u) {
        const float* const p = partial + (int64_t)min(q + 32 * u, blocks - 1) * 2 * F + col;
        va[u] = p[0];
        vb[u] = p[F];
      }
#pragma unroll
      for (int u = 0; u < 4; ++u)
        if (q + 32 * u >= blocks) va[u] = vb[u] = 0.0f;
      a += (va[0] + va[1]) + (va[2] + va[3]);
      b += (vb[0] + vb[1]) + (vb[2] + vb[3]);
    }
  s0[warp][lane] = a;
  s1[warp][lane] = b;
  __syncthreads();
  const int f = blockIdx.x * 32 + warp;
  float S0 = s0[lane][warp], S1 = s1[lane][warp];
#pragma unroll
  for (int d = 16; d > 0; d >>= 1) {
    S0 += __shfl_xor_sync(0xffffffffu, S0, d);
    S1 += __shfl_xor_sync(0xffffffffu, S1, d);
  }
  if (lane != 0 || f >= F) return;
  if (dw_pre) dw_pre[f] = S0;
  if (dw_post) dw_post[f] = gate ? gate[f] * S1 : S1;
  if (dgate) dgate[f] = w_post ? w_post[f] * S1 : S1;
}

constexpr int kMaxF = 8192;
constexpr int kBlocksPerSm = 3;                            // most blocks per SM of the backward kernel (rows of `partial`)

template <typename T, int VEC, int TEAM, int K>
int32_t launch_one(bool backward, const NormArgs& A, int gate_kind, int sms, int* blocks, cudaStream_t st) {
  constexpr int THREADS = TEAM > 256 ? TEAM : 256, TEAMS = THREADS / TEAM;
  const int64_t need = (A.rows + TEAMS - 1) / TEAMS;
  if (!backward) {
    const int64_t most = (int64_t)sms * 32;
    norm_forward<T, VEC, TEAM, K><<<(unsigned)(need < most ? need : most), THREADS, 0, st>>>(A, gate_kind);
    return GNNCO_OK;
  }
  const size_t smem = (size_t)TEAMS * TEAM * K * VEC * sizeof(float);
  const int64_t most = (int64_t)sms * (THREADS > 256 ? 1 : kBlocksPerSm);
  *blocks = (int)(need < most ? need : most);
  norm_backward<T, VEC, TEAM, K><<<*blocks, THREADS, smem, st>>>(A, gate_kind);
  return GNNCO_OK;
}

// Few lanes with several vectors each beat many lanes with one: fewer shuffles per row, and fewer idle lanes where a row is no power
// of two (backward, a vector per lane against this: 1,774,098 x 34 bf16 534 and 208 us, 1,568,659 x 41 float32 504 and 346 us,
// 1.13M x 128 float32 592 and 574 us).  A lane holds at most 16 elements.
template <typename T, int VEC>
int32_t launch_width(bool backward, const NormArgs& A, int gate_kind, int sms, int* blocks, cudaStream_t st) {
  const int v = (A.F + VEC - 1) / VEC;                     // vectors per row
#define GNNCO_NORM(TEAM, K) return launch_one<T, VEC, TEAM, K>(backward, A, gate_kind, sms, blocks, st)
  if (v <= 8) GNNCO_NORM(8, 1);
  if constexpr (VEC <= 2) {
    if (v <= 16) GNNCO_NORM(8, 2);
    if (v <= 24) GNNCO_NORM(8, 3);
    if (v <= 32) GNNCO_NORM(8, 4);
    if (v <= 48) GNNCO_NORM(16, 3);
    if (v <= 64) GNNCO_NORM(16, 4);
    if (v <= 96) GNNCO_NORM(32, 3);
  }
  if constexpr (VEC == 4) {
    if (v <= 16) GNNCO_NORM(8, 2);
    if (v <= 32) GNNCO_NORM(16, 2);
  }
  if (v <= 16) GNNCO_NORM(16, 1);
  if (v <= 32) GNNCO_NORM(32, 1);
  if (v <= 64) GNNCO_NORM(32, 2);
  if constexpr (VEC <= 4) {
    if (v <= 128) GNNCO_NORM(32, 4);
  }
  if constexpr (VEC == 1) {
    if (v <= 256) GNNCO_NORM(32, 8);
    if (v <= 512) GNNCO_NORM(32, 16);
    if (v <= 2048) GNNCO_NORM(256, 8);
    GNNCO_NORM(512, 16);
  } else if constexpr (VEC == 2) {
    if (v <= 256) GNNCO_NORM(32, 8);
    if (v <= 1024) GNNCO_NORM(256, 4);
    GNNCO_NORM(512, 8);
  } else if constexpr (VEC == 4) {
    if (v <= 1024) GNNCO_NORM(256, 4);
    GNNCO_NORM(512, 4);
  } else {
    if (v <= 512) GNNCO_NORM(256, 2);
    GNNCO_NORM(512, 2);
  }
#undef GNNCO_NORM
}

template <typename T>
int32_t launch_typed(bool backward, const NormArgs& A, int gate_kind, int sms, int* blocks, cudaStream_t st) {
  auto fits = [&](int vec) {
    auto ok = [&](const void* p, int64_t ld) { return !p || vec_ok(p, ld, sizeof(T), vec); };
    return A.F % vec == 0 && ok(A.x, A.x_ld) && ok(A.y, A.y_ld) && ok(A.dx_out, A.dx_out_ld) && ok(A.dh, A.dh_ld) &&
           ok(A.x_out, A.x_out_ld) && ok(A.h_out, A.h_out_ld) && ok(A.dx, A.dx_ld) && ok(A.dy, A.dy_ld) &&
           ok(A.dgate, A.dgate_ld) && (gate_kind != kGateRows || ok(A.gate, A.gate_ld));
  };
  if constexpr (sizeof(T) == 2) {
    if (fits(8)) return launch_width<T, 8>(backward, A, gate_kind, sms, blocks, st);
  }
  if (fits(4)) return launch_width<T, 4>(backward, A, gate_kind, sms, blocks, st);
  if (fits(2)) return launch_width<T, 2>(backward, A, gate_kind, sms, blocks, st);
  return launch_width<T, 1>(backward, A, gate_kind, sms, blocks, st);
}

bool valid_block(const gnnco_block_norm_desc* d) {
  if (!d || d->rows < 0 || d->F < 1 || !(d->eps > 0.0f)) return false;
  if (d->gate && d->gate_ld != 0 && d->gate_ld < d->F) return false;
  if (d->rows == 0) return true;                           // empty tensors come without addresses
  if ((d->gate || d->w_post) && !d->y) return false;
  if (d->y && d->y_ld < d->F) return false;
  return d->x_ld >= d->F;
}

NormArgs common_args(const gnnco_block_norm_desc* d) {
  NormArgs A = {};
  A.x = d->x; A.x_ld = d->x_ld;
  A.y = d->y; A.y_ld = d->y_ld;
  A.gate = d->gate; A.gate_ld = d->gate_ld;
  A.w_pre = d->w_pre; A.w_post = d->w_post;
  A.rows = d->rows; A.F = d->F;
  A.scale = d->scale; A.eps = d->eps; A.inv_F = 1.0f / (float)d->F;
  return A;
}
int gate_of(const gnnco_block_norm_desc* d) { return !d->gate ? kGateNone : d->gate_ld == 0 ? kGateVector : kGateRows; }

}  // namespace

extern "C" int32_t gnnco_block_norm(gnnco_handle* h, const gnnco_block_norm_desc* d, void* x_out, int64_t x_out_ld, void* h_out,
                                    int64_t h_out_ld, void* stream) {
  if (!h || !valid_block(d)) return GNNCO_INVALID_ARGUMENT;
  if ((d->feat_dtype != GNNCO_F32 && d->feat_dtype != GNNCO_BF16) || d->F > kMaxF) return GNNCO_UNSUPPORTED;
  if (d->rows == 0) return GNNCO_OK;
  if (!d->x || (!x_out && !h_out) || ((x_out != nullptr) != (d->y != nullptr))) return GNNCO_INVALID_ARGUMENT;
  if ((x_out && x_out_ld < d->F) || (h_out && h_out_ld < d->F)) return GNNCO_INVALID_ARGUMENT;
  cudaStream_t st = static_cast<cudaStream_t>(stream);
  ProfScope prof_(h, K_BLOCK_NORM, st);
  NormArgs A = common_args(d);
  A.x_out = x_out; A.x_out_ld = x_out_ld;
  A.h_out = h_out; A.h_out_ld = h_out_ld;
  int blocks = 0;
  const int32_t rc = d->feat_dtype == GNNCO_F32 ? launch_typed<float>(false, A, gate_of(d), h->sm_count, &blocks, st)
                                                : launch_typed<__nv_bfloat16>(false, A, gate_of(d), h->sm_count, &blocks, st);
  if (rc != GNNCO_OK) return rc;
  h->launches += 1;
  GNNCO_LAUNCH_CHECK();
  return GNNCO_OK;
}

extern "C" int32_t gnnco_block_norm_workspace_bytes(const gnnco_handle* h, int32_t F, size_t* bytes) {
  if (!h || !bytes || F < 1) return GNNCO_INVALID_ARGUMENT;
  *bytes = align_up((size_t)h->sm_count * kBlocksPerSm * 2 * (size_t)F * sizeof(float));
  return GNNCO_OK;
}

extern "C" int32_t gnnco_block_norm_backward(gnnco_handle* h, const gnnco_block_norm_desc* d, const gnnco_block_norm_grads* g,
                                             void* ws, size_t ws_bytes, void* stream) {
  if (!h || !valid_block(d) || !g || !ws || ((uintptr_t)ws & 255)) return GNNCO_INVALID_ARGUMENT;
  if (d->rows > 0) {
    if (!g->dx || g->dx_ld < d->F || (!g->dh && !g->dx_out) || (g->dh && (!d->x || g->dh_ld < d->F)) ||
        (g->dx_out && g->dx_out_ld < d->F))
      return GNNCO_INVALID_ARGUMENT;
    if ((d->y != nullptr) != (g->dy != nullptr) || (g->dy && g->dy_ld < d->F)) return GNNCO_INVALID_ARGUMENT;
    if ((g->dw_post || g->dgate) && !d->y) return GNNCO_INVALID_ARGUMENT;
  }
  const int gate_kind = gate_of(d);
  if (g->dgate && (gate_kind == kGateNone || (gate_kind == kGateRows && g->dgate_ld < d->F))) return GNNCO_INVALID_ARGUMENT;
  if ((d->feat_dtype != GNNCO_F32 && d->feat_dtype != GNNCO_BF16) || d->F > kMaxF) return GNNCO_UNSUPPORTED;
  size_t need = 0;
  gnnco_block_norm_workspace_bytes(h, d->F, &need);
  if (ws_bytes < need) return GNNCO_WORKSPACE_TOO_SMALL;
  cudaStream_t st = static_cast<cudaStream_t>(stream);
  ProfScope prof_(h, K_BLOCK_NORM, st);
  NormArgs A = common_args(d);
  A.dx_out = g->dx_out; A.dx_out_ld = g->dx_out_ld;
  A.dh = g->dh; A.dh_ld = g->dh_ld;
  A.dx = g->dx; A.dx_ld = g->dx_ld;
  A.dy = g->dy; A.dy_ld = g->dy_ld;
  if (gate_kind == kGateRows) { A.dgate = g->dgate; A.dgate_ld = g->dgate_ld; }
  A.partial = static_cast<float*>(ws);
  int blocks = 0;
  if (d->rows > 0) {
    const int32_t rc = d->feat_dtype == GNNCO_F32 ? launch_typed<float>(true, A, gate_kind, h->sm_count, &blocks, st)
                                                  : launch_typed<__nv_bfloat16>(true, A, gate_kind, h->sm_count, &blocks, st);
    if (rc != GNNCO_OK) return rc;
    h->launches += 1;
  }
  float* dgate = gate_kind == kGateVector ? static_cast<float*>(g->dgate) : nullptr;
  if (g->dw_pre || g->dw_post || dgate) {
    norm_weight_sums<<<(d->F + 31) / 32, 1024, 0, st>>>(A.partial, blocks, d->F,
                                                       gate_kind == kGateVector ? static_cast<const float*>(d->gate) : nullptr,
                                                       d->w_post, g->dw_pre, g->dw_post, dgate);
    h->launches += 1;
  }
  GNNCO_LAUNCH_CHECK();
  return GNNCO_OK;
}
