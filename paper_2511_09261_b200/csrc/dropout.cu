// Dropout without a stored mask:  out[r,c] = x[r,c] / (1 - p) where word(r,c) >= p 2^32, else 0  (words: philox.cuh).
// The mask is a function of (seed, layer, step, r, c), so the gradient is the same call on the gradient of out.
//
// A thread takes one vector of 16 bytes (two or four, loaded before the words are computed, took as long or longer: 2.5 M x 256 bfloat16
// 583 us with one, 597 with two, 586 with four).  Elements whose word falls below the limit are set to 0 by selection, not by a
// product: an infinity or NaN that is dropped is gone.
// A quad takes 18 wide products and 19 logical instructions, a quarter of that per element.  In bfloat16, at 4 bytes moved per element,
// this is what bounds it: 4.4 TB/s, the pipe of the wide products 73 % busy, the one of logic and comparisons 55 %; as separate
// high and low products the same work took 647 us.
#include <math.h>

#include "internal.cuh"
#include "mask.cuh"
#include "philox.cuh"
#include "vec_io.cuh"

namespace {

struct DropArgs {
  const void* x;
  void* out;
  int64_t x_ld, out_ld, rows;
  int32_t F;
  int32_t groups;                                          // groups of G columns in a row
  philox::Mask m;
};

__device__ __forceinline__ float pick(uint32_t word, const philox::Mask& m, float v) {
  return word > m.lim ? v * m.scale : 0.0f;
}

// VEC consecutive, aligned elements (4 or 8: whole quads; F is a multiple of VEC).  flat: the rows are one run of elements.
template <typename T, int VEC, int UNROLL, bool FLAT>
__global__ void __launch_bounds__(256) drop_vectors(const __grid_constant__ DropArgs A) {
  const int64_t items = A.rows * A.groups;
  philox::Stream words(A.m);
  for (int64_t base = (int64_t)blockIdx.x * (256 * UNROLL); base < items; base += (int64_t)gridDim.x * (256 * UNROLL)) {
    const int64_t row0 = FLAT ? 0 : base / A.groups;
    const uint32_t rest = FLAT ? 0u : (uint32_t)(base - row0 * A.groups);
    vio::Raw<T, VEC> v[UNROLL];
    int64_t to[UNROLL];
#pragma unroll
    for (int u = 0; u < UNROLL; ++u) {
      const int64_t i = base + u * 256 + threadIdx.x;
      if (i >= items) break;
      int64_t from;
      if (FLAT) {
        from = to[u] = i * VEC;
      } else {
        const uint32_t off = rest + u * 256 + threadIdx.x, r = off / (uint32_t)A.groups, c = off - r * (uint32_t)A.groups;
        from = (row0 + r) * A.x_ld + (int64_t)c * VEC;
        to[u] = (row0 + r) * A.out_ld + (int64_t)c * VEC;
      }
      v[u].template load<true>(static_cast<const T*>(A.x) + from);
    }
#pragma unroll
    for (int u = 0; u < UNROLL; ++u) {
      const int64_t i = base + u * 256 + threadIdx.x;
      if (i >= items) break;
      float f[VEC];
      uint4 w[VEC / 4];                                    // F is a multiple of 4: quads are numbered along the run of groups
      words.quads(A.m, (uint64_t)i * (VEC / 4), w);
#pragma unroll
      for (int k = 0; k < VEC; k += 4) {
        f[k] = pick(w[k / 4].x, A.m, v[u].get(k));
        f[k + 1] = pick(w[k / 4].y, A.m, v[u].get(k + 1));
        f[k + 2] = pick(w[k / 4].z, A.m, v[u].get(k + 2));
        f[k + 3] = pick(w[k / 4].w, A.m, v[u].get(k + 3));
      }
      vio::store_stream<T, VEC>(static_cast<T*>(A.out) + to[u], f);
    }
  }
}

// any width and alignment: UNROLL quads of columns per thread, element by element (100,003 x 99 bfloat16: one quad 19.3 us, two 17.6)
template <typename T, int UNROLL>
__global__ void __launch_bounds__(256) drop_quads(const __grid_constant__ DropArgs A) {
  const int64_t items = A.rows * A.groups;
  philox::Stream words(A.m);
  for (int64_t base = (int64_t)blockIdx.x * (256 * UNROLL); base < items; base += (int64_t)gridDim.x * (256 * UNROLL)) {
    const int64_t row0 = base / A.groups;
    const uint32_t rest = (uint32_t)(base - row0 * A.groups);
    vio::Raw<T, 1> v[UNROLL][4];
    T* to[UNROLL];
    int count[UNROLL];
#pragma unroll
    for (int u = 0; u < UNROLL; ++u) {
      const uint32_t off = rest + u * 256 + threadIdx.x, r = off / (uint32_t)A.groups;
      const int c = (int)(off - r * (uint32_t)A.groups) * 4;
      count[u] = base + u * 256 + threadIdx.x < items ? min(4, A.F - c) : 0;
      const T* const from = static_cast<const T*>(A.x) + (row0 + r) * A.x_ld + c;
      to[u] = static_cast<T*>(A.out) + (row0 + r) * A.out_ld + c;
#pragma unroll
      for (int k = 0; k < 4; ++k)
        if (k < count[u]) v[u][k].template load<true>(from + k);
    }
#pragma unroll
    for (int u = 0; u < UNROLL; ++u) {
      const uint4 w = words.quad(A.m, (uint64_t)(base + u * 256 + threadIdx.x));
      const uint32_t word[4] = {w.x, w.y, w.z, w.w};
#pragma unroll
      for (int k = 0; k < 4; ++k)
        if (k < count[u]) {
          const float f[1] = {pick(word[k], A.m, v[u][k].get(0))};
          vio::store_stream<T, 1>(to[u] + k, f);
        }
    }
  }
}

template <typename T>
void launch_drop(gnnco_handle* h, DropArgs A, cudaStream_t st) {
  constexpr int kVec = 16 / (int)sizeof(T), kUnroll = 1, kQuads = 2;
  auto fits = [&](int vec) {
    const uintptr_t bytes = (uintptr_t)vec * sizeof(T);
    return A.F % vec == 0 && (((uintptr_t)A.x | (uintptr_t)A.out | (uintptr_t)(A.x_ld * (int64_t)sizeof(T)) |
                               (uintptr_t)(A.out_ld * (int64_t)sizeof(T))) % bytes) == 0;
  };
  const bool flat = A.x_ld == A.F && A.out_ld == A.F;
  const int64_t most = (int64_t)h->sm_count * 8;           // eight blocks of 256 threads fill an SM
  auto blocks = [&](int64_t per) {
    const int64_t need = (A.rows * A.groups + per - 1) / per;
    return (unsigned)(need < most ? need : most);
  };
  if (fits(kVec)) {
    A.groups = A.F / kVec;
    if (flat) drop_vectors<T, kVec, kUnroll, true><<<blocks(256 * kUnroll), 256, 0, st>>>(A);
    else drop_vectors<T, kVec, kUnroll, false><<<blocks(256 * kUnroll), 256, 0, st>>>(A);
    return;
  }
  if constexpr (kVec == 8) {
    if (fits(4)) {
      A.groups = A.F / 4;
      if (flat) drop_vectors<T, 4, kUnroll, true><<<blocks(256 * kUnroll), 256, 0, st>>>(A);
      else drop_vectors<T, 4, kUnroll, false><<<blocks(256 * kUnroll), 256, 0, st>>>(A);
      return;
    }
  }
  A.groups = A.F / 4 + (A.F % 4 != 0);                     // (F + 3 may not fit)
  drop_quads<T, kQuads><<<blocks(256 * kQuads), 256, 0, st>>>(A);
}

}  // namespace

bool make_mask(const gnnco_dropout_params* d, philox::Mask* m, bool* drops) {
  if (!(d->p >= 0.0 && d->p <= 1.0)) return false;
  const double limit = nearbyint(d->p * 4294967296.0);     // ties to even, as everywhere
  philox::set_seed(m, d->seed);
  m->step = d->step;
  m->layer = d->layer;
  m->step_dev = d->step_dev;
  *drops = limit >= 1.0;
  m->lim = *drops ? (uint32_t)(limit - 1.0) : 0u;
  m->scale = d->p < 1.0 ? (float)(1.0 / (1.0 - d->p)) : 0.0f;   // p = 1 keeps nothing
  return true;
}

bool on_own_device(const gnnco_handle* h) {
  int device = -1;
  return cudaGetDevice(&device) == cudaSuccess && device == h->device;
}

extern "C" int32_t gnnco_dropout(gnnco_handle* h, int32_t feat_dtype, int64_t rows, int32_t F, const void* x, int64_t x_ld,
                                 const gnnco_dropout_params* d, void* out, int64_t out_ld, void* stream) {
  philox::Mask m;
  bool drops = false;
  if (!h || !d || rows < 0 || F < 1 || !make_mask(d, &m, &drops)) return GNNCO_INVALID_ARGUMENT;
  if (feat_dtype != GNNCO_F32 && feat_dtype != GNNCO_BF16) return GNNCO_UNSUPPORTED;
  if (rows == 0) return GNNCO_OK;
  if (!x || !out || x_ld < F || out_ld < F || rows > ((int64_t)1 << 62) / F || !on_own_device(h)) return GNNCO_INVALID_ARGUMENT;
  if (x == out && x_ld != out_ld && rows > 1) return GNNCO_INVALID_ARGUMENT;         // (a row of out would lie over other rows of x)
  cudaStream_t st = static_cast<cudaStream_t>(stream);
  ProfScope prof_(h, K_DROPOUT, st);
  const size_t es = feat_dtype == GNNCO_F32 ? 4 : 2;
  if (!drops) {                                            // p below 2^-33: 1 / (1 - p) is 1 in float32
    if (x == out) return GNNCO_OK;
    // (rows further apart than a copy in two dimensions takes are few)
    const int64_t most = 0x7fffffff / (int64_t)es;
    if (x_ld <= most && out_ld <= most) {
      GNNCO_CUDA_TRY(cudaMemcpy2DAsync(out, out_ld * es, x, x_ld * es, F * es, rows, cudaMemcpyDeviceToDevice, st));
    } else {
      for (int64_t r = 0; r < rows; ++r)
        GNNCO_CUDA_TRY(cudaMemcpyAsync(static_cast<char*>(out) + r * out_ld * es, static_cast<const char*>(x) + r * x_ld * es, F * es, cudaMemcpyDeviceToDevice, st));
    }
    return GNNCO_OK;
  }
  const DropArgs A = {x, out, x_ld, out_ld, rows, F, 0, m};
  if (feat_dtype == GNNCO_F32) launch_drop<float>(h, A, st);
  else launch_drop<__nv_bfloat16>(h, A, st);
  h->launches += 1;
  GNNCO_LAUNCH_CHECK();
  return GNNCO_OK;
}
