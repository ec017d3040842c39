// The gated feed-forward block of one to four rows with one set of weights (a node evaluated by itself): vector-matrix products,
// bound by the weights' bytes, which are read once (1 x 1,024 x 4,096 bfloat16: 9.6 and 10.5 us from memory, 17 and 8 MB; the launches'
// start and end are most of that).
//
//   rows_product<GATE = true>   h = act(x Wg) .* (x Wu), kept in float32 between the two launches
//   rows_product<GATE = false>  y = drop(h Wd)
//
// A block owns 32 columns of the result and a part of the contraction; its 256 threads split into lanes along the columns (16
// bytes of a row each) and slices along the contraction, every thread with four rows of the weights in flight.  Up to eight blocks, a
// cluster, share the columns: as many as it takes to give every SM a block, since few columns (1,024: 32 blocks) would leave most
// of the memory's bandwidth unused.  The sums of slices, warps and blocks are added in a fixed order, the last ones through
// distributed shared memory.  The second launch overlaps the first (programmatic dependence): it asks for its weights to be brought
// into L2 before it waits for h.
#include "gated_ff.cuh"
#include "tc_common.cuh"
#include "vec_io.cuh"

namespace ff {
namespace {

constexpr int kThreads = 256, kCols = 32;
constexpr int kMostShared = 5120;                          // floats of x or h that a block holds (five blocks fit an SM)

struct RowsArgs {
  const void* x;                                           // GATE: x, else h (float32)
  int64_t x_ld;
  const void *w0, *w1;                                     // Wg and Wu, or Wd
  float* h;
  void* y;
  int64_t y_ld;
  int32_t rows, K, N, per;                                 // per: of K, per block of a cluster
  int32_t act, y_f32, masked;
  philox::Mask mask;
};

template <typename T>
__device__ __forceinline__ float element(const void* p, int64_t i) {
  if constexpr (vio::Is16<T>::value) return __bfloat162float(static_cast<const __nv_bfloat16*>(p)[i]);
  else return static_cast<const float*>(p)[i];
}

// VEC consecutive elements by plain loads (this kernel may have been running while the one before it wrote)
template <typename T, int VEC>
__device__ __forceinline__ void load_plain(vio::Raw<T, VEC>& v, const T* p) {
  if constexpr (VEC * sizeof(T) == 16) {
    const uint4 q = *reinterpret_cast<const uint4*>(p);
    v.w[0] = q.x; v.w[1] = q.y; v.w[2] = q.z; v.w[3] = q.w;
  } else if constexpr (sizeof(T) == 4) {
    v.w[0] = *reinterpret_cast<const uint32_t*>(p);
  } else {
    v.w[0] = *reinterpret_cast<const unsigned short*>(p);
  }
}

// TX: features, TW: weights, R: rows held, VEC: columns per lane
template <bool GATE, typename TX, typename TW, int R, int VEC>
__global__ void __launch_bounds__(kThreads) rows_product(const __grid_constant__ RowsArgs A) {
  constexpr int kLanes = kCols / VEC, kSlices = kThreads / kLanes, kMats = GATE ? 2 : 1, kFlight = 4;
  constexpr bool kRound = vio::Is16<TX>::value && !vio::Is16<TW>::value;      // float32 weights of bfloat16 features
  __shared__ float xs[kMostShared];                        // [R][per]
  __shared__ float warp_sums[8][kMats][R][kCols];
  __shared__ float sums[kMats][R][kCols];
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const uint32_t rank = tc::cluster_ctarank();
  uint32_t ranks;
  asm volatile("mov.u32 %0, %%cluster_nctaid.x;" : "=r"(ranks));
  const int block = blockIdx.x / ranks, c0 = block * kCols;
  const int k0 = (int)rank * A.per, k1 = min(A.K, k0 + A.per);
  const int slice = warp * (32 / kLanes) + lane / kLanes, col = c0 + (lane % kLanes) * VEC;
  const bool in = col < A.N;                               // (VEC divides N)
  const TW* const w0 = static_cast<const TW*>(A.w0) + col;
  const TW* const w1 = static_cast<const TW*>(A.w1) + col;

  if (GATE) {
    asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
  } else {
    if (in && lane % kLanes == 0)
      for (int k = k0 + slice; k < k1; k += kSlices) asm volatile("prefetch.global.L2 [%0];" ::"l"(w0 + (int64_t)k * A.N));
    asm volatile("griddepcontrol.wait;" ::: "memory");
  }
  for (int i = threadIdx.x; i < R * (k1 - k0); i += kThreads) {
    const int r = i / (k1 - k0), k = i - r * (k1 - k0);
    // (h by plain loads: this kernel may have been running while it was written)
    xs[r * A.per + k] = r < A.rows ? (GATE ? element<TX>(A.x, r * A.x_ld + k0 + k) : *((const volatile float*)A.x + r * A.x_ld + k0 + k)) : 0.0f;
  }
  __syncthreads();
  float acc[kMats][R][VEC];
#pragma unroll
  for (int m = 0; m < kMats; ++m)
#pragma unroll
    for (int r = 0; r < R; ++r)
#pragma unroll
      for (int e = 0; e < VEC; ++e) acc[m][r][e] = 0.0f;
  if (in) {
    for (int k = k0 + slice; k < k1; k += kSlices * kFlight) {
      vio::Raw<TW, VEC> w[kFlight][kMats];
#pragma unroll
      for (int i = 0; i < kFlight; ++i)
        if (k + i * kSlices < k1) {
          load_plain(w[i][0], w0 + (int64_t)(k + i * kSlices) * A.N);
          if (GATE) load_plain(w[i][kMats - 1], w1 + (int64_t)(k + i * kSlices) * A.N);
        }
#pragma unroll
      for (int i = 0; i < kFlight; ++i)
        if (k + i * kSlices < k1) {
          float x[R];
#pragma unroll
          for (int r = 0; r < R; ++r) x[r] = xs[r * A.per + k + i * kSlices - k0];
#pragma unroll
          for (int m = 0; m < kMats; ++m)
#pragma unroll
            for (int e = 0; e < VEC; ++e) {
              float v = w[i][m].get(e);
              if (kRound) v = __bfloat162float(__float2bfloat16_rn(v));
#pragma unroll
              for (int r = 0; r < R; ++r) acc[m][r][e] = fmaf(x[r], v, acc[m][r][e]);
            }
        }
    }
  }
#pragma unroll
  for (int m = 0; m < kMats; ++m)
#pragma unroll
    for (int r = 0; r < R; ++r)
#pragma unroll
      for (int e = 0; e < VEC; ++e) {
#pragma unroll
        for (int d = kLanes; d < 32; d <<= 1) acc[m][r][e] += __shfl_xor_sync(0xffffffffu, acc[m][r][e], d);
        if (lane < kLanes) warp_sums[warp][m][r][lane * VEC + e] = acc[m][r][e];
      }
  __syncthreads();
  for (int i = threadIdx.x; i < kMats * R * kCols; i += kThreads) {
    float t = 0.0f;
#pragma unroll
    for (int w = 0; w < 8; ++w) t += (&warp_sums[w][0][0][0])[i];
    (&sums[0][0][0])[i] = t;
  }
  if (ranks > 1) tc::cluster_sync_all();
  else __syncthreads();
  if (rank == 0) {
    for (int i = threadIdx.x; i < R * kCols; i += kThreads) {
      const int r = i / kCols, c = c0 + i % kCols;
      float t[kMats];
#pragma unroll
      for (int m = 0; m < kMats; ++m) {
        t[m] = 0.0f;
        for (uint32_t q = 0; q < ranks; ++q) {
          float v;
          asm volatile("ld.shared::cluster.f32 %0, [%1];" : "=f"(v) : "r"(tc::map_to_cta(tc::smem_u32(&sums[m][0][0] + i), q)) : "memory");
          t[m] += v;
        }
      }
      if (r >= A.rows || c >= A.N) continue;
      if constexpr (GATE) {
        const float g = t[0];
        float a;
        if (A.act == GNNCO_SILU) a = g / (1.0f + expf(-g));
        else if (A.act == GNNCO_GELU) a = 0.5f * g * erfcf(g * -0.70710678f);
        else a = g > 0.0f ? g : (g != g ? g : 0.0f);
        A.h[(int64_t)r * A.N + c] = a * t[kMats - 1];
      } else {
        float v = t[0];
        if (A.masked) {
          philox::Stream words(A.mask);
          const uint4 w = words.quad(A.mask, (uint64_t)r * ((A.N + 3) / 4) + (c >> 2));
          const uint32_t word = (c & 3) == 0 ? w.x : (c & 3) == 1 ? w.y : (c & 3) == 2 ? w.z : w.w;
          v = word > A.mask.lim ? v * A.mask.scale : 0.0f;
        }
        if (A.y_f32) static_cast<float*>(A.y)[r * A.y_ld + c] = v;
        else static_cast<__nv_bfloat16*>(A.y)[r * A.y_ld + c] = __float2bfloat16_rn(v);
      }
    }
  }
  if (ranks > 1) tc::cluster_sync_all();                   // the sums are read before their CTA leaves
}

// blocks of a cluster: a block for every SM
int split_of(int K, int N, int sms) {
  const int blocks = (N + kCols - 1) / kCols;
  int s = 1;
  while (s < 8 && blocks * s < sms && K / (2 * s) >= 64) s *= 2;
  return s;
}

template <bool GATE, typename TX, typename TW, int R, int VEC>
int32_t launch(RowsArgs A, int sms, cudaStream_t st) {
  const int split = split_of(A.K, A.N, sms), blocks = (A.N + kCols - 1) / kCols;
  A.per = (A.K + split - 1) / split;
  cudaLaunchConfig_t cfg{};
  cfg.gridDim = dim3(blocks * split);
  cfg.blockDim = dim3(kThreads);
  cfg.stream = st;
  cudaLaunchAttribute attr[2];
  attr[0].id = cudaLaunchAttributeClusterDimension;
  attr[0].val.clusterDim.x = split; attr[0].val.clusterDim.y = 1; attr[0].val.clusterDim.z = 1;
  attr[1].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr[1].val.programmaticStreamSerializationAllowed = 1;
  cfg.attrs = attr;
  cfg.numAttrs = GATE ? 1 : 2;
  GNNCO_CUDA_TRY(cudaLaunchKernelEx(&cfg, rows_product<GATE, TX, TW, R, VEC>, A));
  return GNNCO_OK;
}
template <bool GATE, typename TX, typename TW, int VEC>
int32_t launch_rows(const RowsArgs& A, int sms, cudaStream_t st) {
  if (A.rows == 1) return launch<GATE, TX, TW, 1, VEC>(A, sms, st);
  if (A.rows == 2) return launch<GATE, TX, TW, 2, VEC>(A, sms, st);
  return launch<GATE, TX, TW, 4, VEC>(A, sms, st);
}
template <bool GATE, typename TX, typename TW>
int32_t launch_vec(const RowsArgs& A, int sms, cudaStream_t st) {
  constexpr int kVec = 16 / (int)sizeof(TW);
  if (A.N % kVec == 0 && (((uintptr_t)A.w0 | (uintptr_t)A.w1) & 15) == 0) return launch_rows<GATE, TX, TW, kVec>(A, sms, st);
  return launch_rows<GATE, TX, TW, 1>(A, sms, st);
}
template <bool GATE>
int32_t launch_typed(const gnnco_gated_ff_desc* d, const RowsArgs& A, int sms, cudaStream_t st) {
  if (d->feat_dtype == GNNCO_F32) return launch_vec<GATE, float, float>(A, sms, st);
  if (d->w_dtype == GNNCO_F32) return launch_vec<GATE, __nv_bfloat16, float>(A, sms, st);
  return launch_vec<GATE, __nv_bfloat16, __nv_bfloat16>(A, sms, st);
}

}  // namespace

// Rows and widths for which these kernels run.  (1,024 x 4,096 x 1,024 bfloat16, device time with cold caches, here and by tiles: one row
// 17.9 and 26.7 us, four 21.6 and 26.0.  More rows' sums do not fit in the registers.)
bool few_rows(const gnnco_gated_ff_desc* d, int sms) {
  if (d->sets != 1 || d->rows < 1 || d->rows > 4) return false;
  const int held = d->rows > 2 ? 4 : (int)d->rows;
  auto fits = [&](int K, int N) {
    const int split = split_of(K, N, sms);
    return (int64_t)held * ((K + split - 1) / split) <= kMostShared;
  };
  return fits(d->F, d->H) && fits(d->H, d->F_out);
}

int32_t launch_few_rows(gnnco_handle* h, const gnnco_gated_ff_desc* d, const philox::Mask* mask, float* hidden, void* y, int64_t y_ld,
                        cudaStream_t st) {
  RowsArgs A = {};
  A.x = d->x; A.x_ld = d->x_ld;
  A.w0 = d->w_gate; A.w1 = d->w_up;
  A.h = hidden;
  A.rows = (int32_t)d->rows; A.K = d->F; A.N = d->H;
  A.act = d->act;
  int32_t rc = launch_typed<true>(d, A, h->sm_count, st);
  if (rc != GNNCO_OK) return rc;
  A.x = hidden; A.x_ld = d->H;
  A.w0 = A.w1 = d->w_down;
  A.y = y; A.y_ld = y_ld;
  A.K = d->H; A.N = d->F_out;
  A.y_f32 = d->feat_dtype == GNNCO_F32;
  if (mask) {
    A.masked = 1;
    A.mask = *mask;
  }
  rc = launch_typed<false>(d, A, h->sm_count, st);
  if (rc == GNNCO_OK) h->launches += 2;
  return rc;
}

}  // namespace ff
