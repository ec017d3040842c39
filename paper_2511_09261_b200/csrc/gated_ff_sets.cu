// The gated feed-forward block in float32 with a set of weights per subgraph of few rows: bound by the weights' bytes, which the tiled
// products would first copy as limbs.  Plain float32 multiplications instead, eight rows of a subgraph at a time:
//
//   set_gates<BACK>   h = act(x Wg) .* (x Wu);  backward also dh = dy' Wd^T, dg, du and, as all of their operands are at hand, the
//                     weight gradients dWg = x^T dg, dWu = x^T du, dWd = h^T dy'
//   set_down          y = drop(h Wd)
//   set_dx            dx = dg Wg^T + du Wu^T
//
// A block owns a subgraph and 32 columns (of h, y or dx); h, dg and du stay in float32 in the work area between two launches.  Products
// along a weight's columns give a lane one column and the warps every eighth row of the contraction; products across them give
// lanes the contraction and a warp four columns.  Every sum has a fixed order.  More than eight rows: the weights come again
// (from L2) for the next eight, and the gradients are added to what the same threads have written.
// What bounds it: multiplications that eight rows do not fill, and loads in flight (backward, 2,000 x 256 x 300 in 300 sets: 218 us for
// 552 MB of weights and gradients, dx 213 for 184 MB).  Rows of x and dy that stand together in shared memory, eight to a column, halved
// its loads (267 us).
#include "gated_ff.cuh"
#include "gated_ff_sets.cuh"

namespace ff {
namespace {

constexpr int kRows = 8, kCols = 32, kDxCols = 32, kThreads = 256, kWarps = kThreads / 32;
constexpr int kMostF = 384, kMostH = 1024;                 // of shared memory: eight rows of x and dy, or of h

// eight rows' values of one column, which stand together
__device__ __forceinline__ void eight(const float* p, float (&v)[kRows]) {
  const float4 a = reinterpret_cast<const float4*>(p)[0], b = reinterpret_cast<const float4*>(p)[1];
  v[0] = a.x; v[1] = a.y; v[2] = a.z; v[3] = a.w;
  v[4] = b.x; v[5] = b.y; v[6] = b.z; v[7] = b.w;
}
__device__ __forceinline__ float warp_sum(float v) {
#pragma unroll
  for (int d = 16; d; d >>= 1) v += __shfl_xor_sync(0xffffffffu, v, d);
  return v;
}

// a = act(g), slope = act'(g)
__device__ __forceinline__ void activate(int act, float g, float& a, float& slope) {
  if (act == GNNCO_SILU) {
    const float s = 1.0f / (1.0f + expf(-g));
    a = g * s;
    slope = fmaf(a, 1.0f - s, s);
  } else if (act == GNNCO_GELU) {
    const float phi = 0.5f * erfcf(g * -0.70710678f);
    a = g * phi;
    slope = fmaf(g * 0.39894228f, expf(-0.5f * g * g), phi);
  } else {
    a = g > 0.0f ? g : (g != g ? g : 0.0f);
    slope = g > 0.0f ? 1.0f : 0.0f;
  }
}

template <bool BACK>
__global__ void __launch_bounds__(kThreads) set_gates(const __grid_constant__ SetArgs A) {
  extern __shared__ __align__(16) float smem[];            // x, dy': [F][kRows], [F_out][kRows]
  __shared__ float part[kWarps][2 * kRows][kCols];         // sums of g and u
  __shared__ float dh[kRows][kCols], h[kRows][kCols], dg[kRows][kCols], du[kRows][kCols];
  float* const xs = smem;
  float* const dys = smem + kRows * A.F;
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const int64_t set = blockIdx.x / A.h_blocks;
  const int c0 = (int)(blockIdx.x - set * A.h_blocks) * kCols, col = c0 + lane;
  const int begin = A.part_ptr[set], end = A.part_ptr[set + 1];
  const bool in = col < A.H;
  const float *const wg = A.wg + set * A.F * A.H, *const wu = A.wu + set * A.F * A.H, *const wd = A.wd + set * A.H * A.F_out;
  philox::Stream words(A.mask);
  // (a subgraph without rows takes one round of none: its gradients are zeros)
  for (int r0 = begin; r0 == begin || r0 < end; r0 += kRows) {
    const int rows = min(kRows, end - r0);
    __syncthreads();
    for (int i = threadIdx.x; i < kRows * A.F; i += kThreads) {
      const int r = i / A.F;
      xs[(i - r * A.F) * kRows + r] = r < rows ? A.x[(int64_t)(r0 + r) * A.x_ld + i - r * A.F] : 0.0f;
    }
    if (BACK) {
      const int quads = (A.F_out + 3) / 4;
      for (int i = threadIdx.x; i < kRows * quads; i += kThreads) {
        const int r = i / quads, o = (i - r * quads) * 4;
        uint4 w = make_uint4(~0u, ~0u, ~0u, ~0u);
        if (A.masked) w = words.quad(A.mask, (uint64_t)(r0 + r) * quads + o / 4);
        const uint32_t word[4] = {w.x, w.y, w.z, w.w};
#pragma unroll
        for (int e = 0; e < 4; ++e)
          if (o + e < A.F_out) {
            float v = r < rows ? A.dy[(int64_t)(r0 + r) * A.dy_ld + o + e] : 0.0f;
            if (A.masked) v = word[e] > A.mask.lim ? v * A.mask.scale : 0.0f;
            dys[(o + e) * kRows + r] = v;
          }
      }
    }
    __syncthreads();
    float g[kRows] = {}, u[kRows] = {};
    if (in) {
#pragma unroll 4
      for (int k = warp; k < A.F; k += kWarps) {
        const float a = wg[(int64_t)k * A.H + col], b = wu[(int64_t)k * A.H + col];
        float x[kRows];
        eight(xs + k * kRows, x);
#pragma unroll
        for (int r = 0; r < kRows; ++r) {
          g[r] = fmaf(x[r], a, g[r]);
          u[r] = fmaf(x[r], b, u[r]);
        }
      }
    }
#pragma unroll
    for (int r = 0; r < kRows; ++r) {
      part[warp][r][lane] = g[r];
      part[warp][kRows + r][lane] = u[r];
    }
    if (BACK) {
#pragma unroll
      for (int j = 0; j < kCols / kWarps; ++j) {
        const int c = warp * (kCols / kWarps) + j;
        float s[kRows] = {};
        if (c0 + c < A.H)
          for (int o = lane; o < A.F_out; o += 32) {
            const float w = wd[(int64_t)(c0 + c) * A.F_out + o];
            float y[kRows];
            eight(dys + o * kRows, y);
#pragma unroll
            for (int r = 0; r < kRows; ++r) s[r] = fmaf(y[r], w, s[r]);
          }
#pragma unroll
        for (int r = 0; r < kRows; ++r) {
          s[r] = warp_sum(s[r]);
          if (lane == 0) dh[r][c] = s[r];
        }
      }
    }
    __syncthreads();
    {
      const int r = warp;                                  // (a row per warp, a column per lane)
      float gs = 0.0f, us = 0.0f, a, slope;
#pragma unroll
      for (int w = 0; w < kWarps; ++w) {
        gs += part[w][r][lane];
        us += part[w][kRows + r][lane];
      }
      activate(A.act, gs, a, slope);
      const bool valid = r < rows && in;
      const int64_t at = (int64_t)(r0 + r) * A.H + col;
      h[r][lane] = valid ? a * us : 0.0f;
      if (!BACK && valid) A.h[at] = a * us;
      if (BACK) {
        const float d = dh[r][lane];
        dg[r][lane] = valid ? d * us * slope : 0.0f;
        du[r][lane] = valid ? d * a : 0.0f;
        if (valid && A.dg) {
          A.dg[at] = dg[r][lane];
          A.du[at] = du[r][lane];
        }
      }
    }
    if (BACK && A.dwg) {
      __syncthreads();
      float dgr[kRows], dur[kRows];
#pragma unroll
      for (int r = 0; r < kRows; ++r) {
        dgr[r] = dg[r][lane];
        dur[r] = du[r][lane];
      }
      if (in) {
        for (int k = warp; k < A.F; k += kWarps) {
          const int64_t at = (set * A.F + k) * A.H + col;
          float sg = r0 == begin ? 0.0f : A.dwg[at], su = r0 == begin ? 0.0f : A.dwu[at];
          float x[kRows];
          eight(xs + k * kRows, x);
#pragma unroll
          for (int r = 0; r < kRows; ++r) {
            sg = fmaf(x[r], dgr[r], sg);
            su = fmaf(x[r], dur[r], su);
          }
          A.dwg[at] = sg;
          A.dwu[at] = su;
        }
      }
      for (int j = 0; j < kCols / kWarps; ++j) {
        const int c = warp * (kCols / kWarps) + j;
        if (c0 + c >= A.H) break;
        float hr[kRows];
#pragma unroll
        for (int r = 0; r < kRows; ++r) hr[r] = h[r][c];
        for (int o = lane; o < A.F_out; o += 32) {
          const int64_t at = (set * A.H + c0 + c) * A.F_out + o;
          float s = r0 == begin ? 0.0f : A.dwd[at];
          float y[kRows];
          eight(dys + o * kRows, y);
#pragma unroll
          for (int r = 0; r < kRows; ++r) s = fmaf(hr[r], y[r], s);
          A.dwd[at] = s;
        }
      }
    }
  }
}

__global__ void __launch_bounds__(kThreads) set_down(const __grid_constant__ SetArgs A) {
  extern __shared__ __align__(16) float hs[];              // [H][kRows]
  __shared__ float part[kWarps][kRows][kCols];
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const int64_t set = blockIdx.x / A.out_blocks;
  const int col = (int)(blockIdx.x - set * A.out_blocks) * kCols + lane;
  const int begin = A.part_ptr[set], end = A.part_ptr[set + 1];
  const bool in = col < A.F_out;
  const float* const wd = A.wd + set * A.H * A.F_out;
  philox::Stream words(A.mask);
  for (int r0 = begin; r0 < end; r0 += kRows) {
    const int rows = min(kRows, end - r0);
    __syncthreads();
    for (int i = threadIdx.x; i < kRows * A.H; i += kThreads) {
      const int r = i / A.H;
      hs[(i - r * A.H) * kRows + r] = r < rows ? A.h[(int64_t)r0 * A.H + i] : 0.0f;
    }
    __syncthreads();
    float s[kRows] = {};
    if (in) {
#pragma unroll 4
      for (int k = warp; k < A.H; k += kWarps) {
        const float w = wd[(int64_t)k * A.F_out + col];
        float v[kRows];
        eight(hs + k * kRows, v);
#pragma unroll
        for (int r = 0; r < kRows; ++r) s[r] = fmaf(v[r], w, s[r]);
      }
    }
#pragma unroll
    for (int r = 0; r < kRows; ++r) part[warp][r][lane] = s[r];
    __syncthreads();
    if (warp < rows && in) {
      float v = 0.0f;
#pragma unroll
      for (int w = 0; w < kWarps; ++w) v += part[w][warp][lane];
      if (A.masked) {
        const uint4 w = words.quad(A.mask, (uint64_t)(r0 + warp) * ((A.F_out + 3) / 4) + (col >> 2));
        const uint32_t word = (col & 3) == 0 ? w.x : (col & 3) == 1 ? w.y : (col & 3) == 2 ? w.z : w.w;
        v = word > A.mask.lim ? v * A.mask.scale : 0.0f;
      }
      A.out[(int64_t)(r0 + warp) * A.out_ld + col] = v;
    }
  }
}

__global__ void __launch_bounds__(kThreads) set_dx(const __grid_constant__ SetArgs A) {
  constexpr int kEach = kDxCols / kWarps;                  // columns of a warp
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const int64_t set = blockIdx.x / A.out_blocks;
  const int c0 = (int)(blockIdx.x - set * A.out_blocks) * kDxCols + warp * kEach;
  const int begin = A.part_ptr[set], end = A.part_ptr[set + 1];
  const float *const wg = A.wg + (set * A.F + c0) * A.H, *const wu = A.wu + (set * A.F + c0) * A.H;
  for (int r0 = begin; r0 < end; r0 += kRows) {
    const int rows = min(kRows, end - r0);
    float s[kEach][kRows] = {};
    for (int k = lane; k < A.H; k += 32) {
      float a[kRows], b[kRows];
#pragma unroll
      for (int r = 0; r < kRows; ++r) {
        a[r] = r < rows ? A.dg[(int64_t)(r0 + r) * A.H + k] : 0.0f;
        b[r] = r < rows ? A.du[(int64_t)(r0 + r) * A.H + k] : 0.0f;
      }
#pragma unroll
      for (int j = 0; j < kEach; ++j)
        if (c0 + j < A.F) {
          const float p = wg[(int64_t)j * A.H + k], q = wu[(int64_t)j * A.H + k];
#pragma unroll
          for (int r = 0; r < kRows; ++r) s[j][r] = fmaf(a[r], p, fmaf(b[r], q, s[j][r]));
        }
    }
#pragma unroll
    for (int j0 = 0; j0 < kEach; j0 += 4) {                // lane (r, j) keeps one of 32 sums
      float mine = 0.0f;
#pragma unroll
      for (int j = 0; j < 4; ++j)
#pragma unroll
        for (int r = 0; r < kRows; ++r) {
          const float v = warp_sum(s[j0 + j][r]);
          if (lane == r * 4 + j) mine = v;
        }
      const int r = lane / 4, c = c0 + j0 + lane % 4;
      if (r < rows && c < A.F) A.out[(int64_t)(r0 + r) * A.out_ld + c] = mine;
    }
  }
}

}  // namespace

// (Whole calls, here and by tiles of limbs, us: backward 2,000 x 256 x 300 in 300 sets 431 and 482, 1,292 x 20 x 596 in 585 267 and 492,
// 4,301 x 26 x 541 in 882 388 and 611; forward 326 x 198 x 477 in 163 113 and 177, 1,729 x 52 x 504 in 261 60 and 95; but with more rows
// than eight on average 12,000 x 237 x 258 in 934 backward 2,171 and 1,266, 8,755 x 230 x 285 in 676 forward 447 and 456.)
bool few_rows_per_set(const gnnco_handle* h, const gnnco_gated_ff_desc* d) {
  return d->feat_dtype == GNNCO_F32 && d->sets > 1 && d->F <= kMostF && d->F_out <= kMostF && d->H <= kMostH && h->longest_part <= 8 * kRows &&
         d->rows <= kRows * (int64_t)d->sets;
}

int32_t launch_sets(gnnco_handle* h, SetArgs A, int64_t sets, bool backward, cudaStream_t st) {
  A.part_ptr = h->part_ptr;
  A.h_blocks = (A.H + kCols - 1) / kCols;
  const int64_t gates = sets * A.h_blocks;
  A.out_blocks = backward ? (A.F + kDxCols - 1) / kDxCols : (A.F_out + kCols - 1) / kCols;
  const int64_t outs = sets * A.out_blocks;
  if (gates > 0x7fffffff || outs > 0x7fffffff) return GNNCO_UNSUPPORTED;
  const size_t held = (size_t)kRows * (A.F + A.F_out) * 4;
  if (backward) {
    set_gates<true><<<(unsigned)gates, kThreads, held, st>>>(A);
    if (A.out) set_dx<<<(unsigned)outs, kThreads, 0, st>>>(A);
  } else {
    set_gates<false><<<(unsigned)gates, kThreads, held, st>>>(A);
    set_down<<<(unsigned)outs, kThreads, (size_t)kRows * A.H * 4, st>>>(A);
  }
  h->launches += backward && !A.out ? 1 : 2;
  return GNNCO_OK;
}

}  // namespace ff
