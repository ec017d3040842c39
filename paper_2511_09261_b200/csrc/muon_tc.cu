// Newton-Schulz iterations of matrices of up to 256 x 256 that never leave the chip: one CTA (short side up to 128) or a
// pair of CTAs (cluster of two, cta_group::2) takes a matrix from gradient to updated weight.
//
// Per step three products run on the tensor cores, X being k x n (padded with zeros):
//   A = X X^T        both operands from shared memory (rows of X, k-major)
//   A A              left operand from tensor memory, right one from shared memory (A is symmetric: its rows)
//   X' = P X         P = a I + b A + c A A from tensor memory, X from shared memory (n-major: the same bytes)
//
// Accuracy.  Operands are float16 pairs (limbs): x = hi + lo with hi = fl16(x), lo = fl16(x - hi), 22 bits together, at
// power-of-two scales that keep hi in range and lo normal; a product is hi hi + hi lo + lo hi (the dropped lo lo is
// 2^-24 of it) summed in the float32 accumulator.  The tensor core drops the bits below the accumulator's last place at
// every instruction, so the small products of all k come first and the large ones meet the accumulator only k / 16
// times (error of a 256 x 256 iterate after 5 steps: 8.1e-6 interleaved; see below for this order).  That is float32
// accuracy at a third of the float16 rate; one float16 or bfloat16 product would put 2e-3 (1.5e-2) into the result, because errors in the direction of small singular values
// grow by a = 3.4 per step.
//
// Where things live.  Shared memory: X in two limbs (panels of 64 columns, 128 rows of 128 bytes, 128-byte swizzle: the same
// bytes serve as k-major rows and as n-major columns) and A's limbs.  Tensor memory, in blocks of 32 columns: the
// accumulator of X X^T is replaced in place by A's limbs (16 + 16 columns) and those by P's; a second accumulator
// takes A A and then X'.
//
// A pair: each CTA owns 128 rows of X, A, P and of the accumulators.  X X^T and A A need only own rows as right operand
// (half of N each); P X needs X by column halves, so after X X^T each CTA replaces its off-diagonal 128 x 128 block of X by
// the partner's, which the partner left in a global scratch line (L2) when it wrote its rows -- both are copied in while
// A and A A are worked on.  A's low limb does not fit next to X as a whole: its second half follows into the room of the
// first as soon as the products that read the first are done (they are issued first).
//
// Roles: warp 16 issues MMAs and the exchange; warps 0-15 load, convert and store: warp w owns rows 32 (w % 4) .. +32 (its TMEM
// lanes) and the 32-column items w / 4 and w / 4 + 4.  Barriers per 64-column panel let the next product start on the
// first panels while the others are converted.  Every wait is bounded; a CTA that gives up raises the status word.
#include <cuda_fp16.h>
#include <math.h>

#include "muon_internal.cuh"
#include "tc_common.cuh"
#include "vec_io.cuh"

namespace {

constexpr int kWorkWarps = 16, kThreads = 32 * (kWorkWarps + 1);
constexpr uint32_t kPanel = 16384;                         // 128 rows x 64 float16
constexpr float kXScale = 16384.0f;                        // |X| <= 2 on entry and by the bound on the coefficients
constexpr float kAScale = 8192.0f;                         // |A| <= 4

template <bool PAIR>
struct Cfg {
  static constexpr int CTAS = PAIR ? 2 : 1;
  static constexpr uint32_t X_BYTES = 2 * 4 * kPanel;
  static constexpr int A_HI = PAIR ? 4 : 2, A_LO = 2;      // panels of A's limbs in shared memory
  static constexpr uint32_t A_BYTES = (A_HI + A_LO) * kPanel;
  static constexpr uint32_t MISC = 1024;
  static constexpr size_t SMEM = 1024 + X_BYTES + A_BYTES + MISC;
  static constexpr uint32_t ACC1 = 0, ACC2 = PAIR ? 256 : 128, ACC3 = 256;   // TMEM columns
  static_assert(SMEM <= 232448, "does not fit in shared memory");
};

struct Bars {
  uint64_t x[4], a[4], p[4];                               // panel ready (used in the even CTA)
  uint64_t m1, m2, m3, lofree;                             // products done (both CTAs)
  uint64_t l;                                              // second half of A's low limb ready (even CTA)
  uint64_t g, s, s2;                                       // partner's block in scratch / copied here / copied there
  uint64_t norm, norm2, loaded;                            // loader: sums ready, partner's sum ready, X written
};

__device__ __forceinline__ uint32_t pack_f16(float lo, float hi) {
  uint32_t r;
  asm("cvt.rn.f16x2.f32 %0, %1, %2;" : "=r"(r) : "f"(hi), "f"(lo));
  return r;
}
__device__ __forceinline__ float2 unpack_f16(uint32_t v) { return __half22float2(*reinterpret_cast<__half2*>(&v)); }
// x, y -> packed high limbs and packed low limbs
__device__ __forceinline__ void split2(float x, float y, uint32_t& hi, uint32_t& lo) {
  hi = pack_f16(x, y);
  const float2 f = unpack_f16(hi);
  lo = pack_f16(x - f.x, y - f.y);
}
// row r, 16-byte chunk c of a panel
__device__ __forceinline__ uint32_t at_chunk(int r, int c) { return (uint32_t)(r * 128 + ((c ^ (r & 7)) << 4)); }

template <bool PAIR>
struct Waiter {
  volatile uint32_t* abort_flag;
  __device__ __forceinline__ bool operator()(uint64_t* bar, uint32_t parity) const {
    auto ready = [&]() { return PAIR ? tc::mbar_try_wait_cluster(bar, parity) : tc::mbar_try_wait(bar, parity); };
    if (ready()) return true;
    const long long t0 = clock64();
    while (!ready()) {
      if (*abort_flag) return false;
      if (clock64() - t0 > 4000000000ll) {
        *abort_flag = 1;
        return false;
      }
    }
    return true;
  }
};

template <bool PAIR>
__global__ void __launch_bounds__(kThreads, 1) ns_on_chip(const NsJob J) {
  using C = Cfg<PAIR>;
  extern __shared__ uint8_t smem_raw[];
  const uint32_t sbase = (tc::smem_u32(smem_raw) + 1023u) & ~1023u;
  const uint32_t sX = sbase, sA = sbase + C::X_BYTES;
  uint8_t* gen = smem_raw + (sbase - tc::smem_u32(smem_raw));
  Bars* B = reinterpret_cast<Bars*>(gen + C::X_BYTES + C::A_BYTES);
  uint32_t* tmem_slot = reinterpret_cast<uint32_t*>(B + 1);
  volatile uint32_t* abort_flag = tmem_slot + 1;
  double* sums = reinterpret_cast<double*>(gen + C::X_BYTES + C::A_BYTES + 512);   // [16] own warps, [16 + rank] per CTA

  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const uint32_t rank = PAIR ? tc::cluster_ctarank() : 0u;
  const int64_t group = blockIdx.x / C::CTAS, groups = gridDim.x / C::CTAS;
  const int kc = (J.k + 15) / 16 * 16, nc = (J.n + 15) / 16 * 16;   // contraction lengths
  const int a_items = (kc + 31) / 32, x_items = (nc + 31) / 32;     // 32-column items of A / P and of X
  const int quarters = PAIR ? 4 : (J.k + 31) / 32;                  // row quarters that hold anything
  const Waiter<PAIR> wait{abort_flag};

  if (threadIdx.x == 0) {
    auto panel_items = [](int items, int p) { const int left = items - 2 * p; return left <= 0 ? 1 : left >= 2 ? 2 : left; };
    for (int p = 0; p < 4; ++p) {
      tc::mbar_init(&B->x[p], quarters * panel_items(x_items, p) * C::CTAS);
      tc::mbar_init(&B->a[p], quarters * panel_items(a_items, p) * C::CTAS);
      tc::mbar_init(&B->p[p], quarters * panel_items(a_items, p) * C::CTAS);
    }
    tc::mbar_init(&B->m1, 1); tc::mbar_init(&B->m2, 1); tc::mbar_init(&B->m3, 1); tc::mbar_init(&B->lofree, 1);
    tc::mbar_init(&B->l, 4 * (a_items > 4 ? a_items - 4 : 1) * C::CTAS);
    // items of the partner's off-diagonal half: the odd CTA receives the even one's upper columns and vice versa
    const int off_items = rank == 1 ? (x_items > 4 ? x_items - 4 : 1) : 4;
    tc::mbar_init(&B->g, 4 * off_items);
    tc::mbar_init(&B->s, 1); tc::mbar_init(&B->s2, 1);
    tc::mbar_init(&B->norm, kWorkWarps); tc::mbar_init(&B->norm2, 1); tc::mbar_init(&B->loaded, kWorkWarps);
    *abort_flag = 0;
    tc::fence_mbar_init();
  }
  if (warp == 0) {
    if constexpr (PAIR) tc::tmem_alloc_pair(tmem_slot, 512);
    else tc::tmem_alloc(tmem_slot, 512);
  }
  tc::tc_fence_before_sync();
  __syncthreads();
  if constexpr (PAIR) tc::cluster_sync_all();
  tc::tc_fence_after_sync();
  const uint32_t tmem = *tmem_slot;
  // the exchange scratch of this pair: [CTA][limb][2 panels]
  uint8_t* const scratch = PAIR ? static_cast<uint8_t*>(J.scratch) + group * (2 * 4 * (int64_t)kPanel) : nullptr;

  if (warp == kWorkWarps) {
    // ------------------------------------------------------------------------------ MMA issue, exchange
    if (lane == 0) {
      const uint32_t i1 = tc::idesc_f16_f32(PAIR ? 256 : 128, PAIR ? 256 : kc, false);
      const uint32_t i3 = tc::idesc_f16_f32(PAIR ? 256 : 128, PAIR ? 256 : nc, true);
      auto commit = [&](uint64_t* bar) {
        if constexpr (PAIR) tc::mma_commit_pair(bar, 3);
        else tc::mma_commit(bar);
      };
      auto left = [&](int t, int limb) { return (uint64_t)(tmem + C::ACC1 + (t >> 1) * 32 + (t & 1) * 8 + limb * 16); };
      auto kmajor = [&](uint32_t base, int t) { return tc::smem_desc_sw128(base + (t >> 2) * kPanel + (t & 3) * 32, 16, 1024); };
      // rows 16 t .. of X: in a pair rows 128 .. are in panels 2 and 3
      auto nmajor = [&](uint32_t base, int t) {
        const uint32_t off = PAIR ? (uint32_t)(t >> 3) * 2 * kPanel + (uint32_t)(t & 7) * 2048u : (uint32_t)t * 2048u;
        return tc::smem_desc_sw128(base + off, kPanel, 1024);
      };
      const uint32_t xh = sX, xl = sX + 4 * kPanel, ah = sA, al = sA + C::A_HI * kPanel;
      const int tk = kc / 16, tn = nc / 16;                // k-steps of 16
      uint32_t it = 0;
      for (int64_t s = group; s < J.sets && !*abort_flag; s += groups) {
        if (J.active && !J.active[s]) continue;
        for (int step = 0; step < J.steps; ++step, ++it) {
          const uint32_t ph = it & 1;
          if (rank == 0) {
            for (int t = 0; t < tn; ++t) {                 // X X^T
              if ((t & 3) == 0) {
                if (!wait(&B->x[t >> 2], ph)) break;
                tc::tc_fence_after_sync();
              }
              tc::mma_f16<PAIR, false>(tmem + C::ACC1, kmajor(xh, t), kmajor(xl, t), i1, t != 0);
              tc::mma_f16<PAIR, false>(tmem + C::ACC1, kmajor(xl, t), kmajor(xh, t), i1, true);
            }
            for (int t = 0; t < tn; ++t) tc::mma_f16<PAIR, false>(tmem + C::ACC1, kmajor(xh, t), kmajor(xh, t), i1, true);
            commit(&B->m1);
          }
          if constexpr (PAIR) {
            // X X^T has read the rows; the off-diagonal block gives way to the partner's
            if (!wait(&B->m1, ph) || !wait(&B->g, ph)) break;
            tc::fence_proxy_async_all();
            tc::mbar_arrive_expect_tx(&B->s, 4 * kPanel);
            const uint8_t* from = scratch + (rank ^ 1u) * 4 * kPanel;
            for (int limb = 0; limb < 2; ++limb)
              tc::bulk_load((limb ? xl : xh) + (rank == 0 ? 2 : 0) * kPanel, from + limb * 2 * kPanel, 2 * kPanel, &B->s);
            if (rank == 1) {
              if (!wait(&B->s, ph)) break;
              tc::mbar_arrive_release_cluster(tc::map_to_cta(tc::smem_u32(&B->s2), 0));
            }
          }
          if (rank == 0) {
            bool ok = true;                                // A A
            if constexpr (PAIR) {
              for (int t = 0; t < 8 && ok; ++t) {          // what reads the first half of A's low limb comes first
                if ((t & 3) == 0) {
                  ok = wait(&B->a[t >> 2], ph);
                  tc::tc_fence_after_sync();
                }
                if (ok) tc::mma_f16<true, true>(tmem + C::ACC2, left(t, 0), kmajor(al, t), i1, t != 0);
              }
              if (!ok) break;
              commit(&B->lofree);
            }
            for (int t = 0; t < tk && ok; ++t) {
              if ((t & 3) == 0 && !(PAIR && t < 8)) {
                ok = wait(&B->a[t >> 2], ph);
                tc::tc_fence_after_sync();
              }
              if (!ok) break;
              tc::mma_f16<PAIR, true>(tmem + C::ACC2, left(t, 1), kmajor(ah, t), i1, PAIR || t != 0);
              if constexpr (!PAIR) tc::mma_f16<PAIR, true>(tmem + C::ACC2, left(t, 0), kmajor(al, t), i1, true);
            }
            if constexpr (PAIR) {
              if (!ok || !wait(&B->l, ph)) break;
              tc::tc_fence_after_sync();
              for (int t = 8; t < tk; ++t) tc::mma_f16<true, true>(tmem + C::ACC2, left(t, 0), kmajor(al, t - 8), i1, true);
            }
            for (int t = 0; t < tk && ok; ++t) tc::mma_f16<PAIR, true>(tmem + C::ACC2, left(t, 0), kmajor(ah, t), i1, true);
            if (!ok) break;
            commit(&B->m2);
            // P X.  In a pair the accumulator is the one A A is read from: all of P must be there.
            if constexpr (PAIR) {
              for (int p = 0; 64 * p < kc; ++p) ok = ok && wait(&B->p[p], ph);
              ok = ok && wait(&B->s, ph) && wait(&B->s2, ph);
              tc::tc_fence_after_sync();
            }
            for (int t = 0; t < tk && ok; ++t) {
              if (!PAIR && (t & 3) == 0) {
                ok = wait(&B->p[t >> 2], ph);
                tc::tc_fence_after_sync();
                if (!ok) break;
              }
              tc::mma_f16<PAIR, true>(tmem + C::ACC3, left(t, 0), nmajor(xl, t), i3, t != 0);
              tc::mma_f16<PAIR, true>(tmem + C::ACC3, left(t, 1), nmajor(xh, t), i3, true);
            }
            for (int t = 0; t < tk && ok; ++t) tc::mma_f16<PAIR, true>(tmem + C::ACC3, left(t, 0), nmajor(xh, t), i3, true);
            if (!ok) break;
            commit(&B->m3);
          }
        }
      }
    }
    __syncwarp();
  } else {
    // ------------------------------------------------------------------------------ load, convert, store
    const int quarter = warp & 3, sub = warp >> 2;
    const int row = quarter * 32 + lane;                   // of this CTA's 128
    const uint32_t lanes = (uint32_t)(quarter * 32) << 16;
    const int grow = (int)rank * 128 + row;                // row of X
    const bool works = quarter < quarters;
    const int off_panel = rank == 0 ? 2 : 0;               // the two panels that the partner takes
    auto arrive = [&](uint64_t* bar) {                     // on the even CTA's barrier, by one lane, after __syncwarp
      if constexpr (PAIR) tc::mbar_arrive_release_cluster(tc::map_to_cta(tc::smem_u32(bar), 0));
      else tc::mbar_arrive(bar);
    };
    // the items of X that this warp owns are written: tell the issuer, and the partner about its share of the scratch
    auto x_ready = [&](int item) {
      if (works && item < x_items && lane == 0) arrive(&B->x[item >> 1]);
    };
    auto partner_ready = [&](int item) {
      if (PAIR && item < x_items && ((item >> 1) & 2) == off_panel && lane == 0) {
        __threadfence();
        tc::mbar_arrive_release_cluster(tc::map_to_cta(tc::smem_u32(&B->g), rank ^ 1u));
      }
    };
    auto put_chunk = [&](int limb, int r, int chunk, uint32_t v0, uint32_t v1, uint32_t v2, uint32_t v3) {
      // chunk: 8 columns, counted over the row
      const int panel = chunk >> 3;
      const uint32_t o = at_chunk(r, chunk & 7);
      tc::st_shared16(sX + (limb * 4 + panel) * kPanel + o, v0, v1, v2, v3);
      if (PAIR && (panel & 2) == off_panel)
        *reinterpret_cast<uint4*>(scratch + rank * 4 * kPanel + (limb * 2 + (panel & 1)) * kPanel + o) = make_uint4(v0, v1, v2, v3);
    };
    const int cpr = (nc + 31) / 32 * 4;                    // chunks per row that are kept (whole items)
    const int rows_kept = quarters * 32, total = rows_kept * cpr;
    uint32_t it = 0, mat = 0;
    for (int64_t s = group; s < J.sets && !*abort_flag; s += groups) {
      if (J.active && !J.active[s]) continue;
      const int64_t base = s * (int64_t)J.r * J.c;
      // ---- momentum, u, |u|^2: eight chunks of eight columns per thread
      float u[8][8];
      double sum = 0.0;
#pragma unroll
      for (int z = 0; z < 8; ++z) {
        const int q = threadIdx.x + z * (32 * kWorkWarps);
        int r, ch;
        if (J.transpose) { ch = q / rows_kept; r = q - ch * rows_kept; }
        else { r = q / cpr; ch = q - r * cpr; }
        const int i = (int)rank * 128 + r, j0 = ch * 8;
        const bool in = q < total && i < J.k && j0 < J.n;
        if (in && J.vec4) {                                // four float32 columns at a time (rows are 16-byte aligned)
#pragma unroll
          for (int hf = 0; hf < 2; ++hf) {
            const int64_t at = base + (int64_t)i * J.c + j0 + 4 * hf;
            float4 g = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
            if (j0 + 4 * hf < J.n) {
              g = __ldcs(reinterpret_cast<const float4*>(static_cast<const float*>(J.G) + at));
              if (J.m) {
                float4 mv = *reinterpret_cast<const float4*>(J.m + at);
                mv.x = J.mu * mv.x + g.x; mv.y = J.mu * mv.y + g.y; mv.z = J.mu * mv.z + g.z; mv.w = J.mu * mv.w + g.w;
                *reinterpret_cast<float4*>(J.m + at) = mv;
                if (J.nesterov) { g.x += J.mu * mv.x; g.y += J.mu * mv.y; g.z += J.mu * mv.z; g.w += J.mu * mv.w; }
                else g = mv;
              }
            }
            u[z][4 * hf] = g.x; u[z][4 * hf + 1] = g.y; u[z][4 * hf + 2] = g.z; u[z][4 * hf + 3] = g.w;
          }
        } else {
#pragma unroll
          for (int e = 0; e < 8; ++e) {
            float v = 0.0f;
            if (in && j0 + e < J.n) {
              const int64_t at = base + (J.transpose ? (int64_t)(j0 + e) * J.c + i : (int64_t)i * J.c + j0 + e);
              v = J.g_bf16 ? __bfloat162float(static_cast<const __nv_bfloat16*>(J.G)[at]) : __ldcs(static_cast<const float*>(J.G) + at);
              if (J.m) {
                const float mv = J.mu * J.m[at] + v;
                J.m[at] = mv;
                v = J.nesterov ? v + J.mu * mv : mv;
              }
            }
            u[z][e] = v;
          }
        }
#pragma unroll
        for (int e = 0; e < 8; ++e) sum += (double)u[z][e] * (double)u[z][e];
      }
#pragma unroll
      for (int d = 16; d > 0; d >>= 1) sum += __shfl_xor_sync(0xffffffffu, sum, d);
      if (lane == 0) {
        sums[warp] = sum;
        tc::mbar_arrive(&B->norm);
      }
      if (!wait(&B->norm, mat & 1)) break;
      double norm2 = 0.0;
#pragma unroll
      for (int w = 0; w < kWorkWarps; ++w) norm2 += sums[w];
      if constexpr (PAIR) {
        if (threadIdx.x == 0) {
          const uint32_t peer = tc::map_to_cta(tc::smem_u32(sums + 16), rank ^ 1u);
          asm volatile("st.shared::cluster.f64 [%0], %1;" ::"r"(peer), "d"(norm2) : "memory");
          tc::mbar_arrive_release_cluster(tc::map_to_cta(tc::smem_u32(&B->norm2), rank ^ 1u));
        }
        if (!wait(&B->norm2, mat & 1)) break;
        norm2 += sums[16];                                 // a + b = b + a: both CTAs get the same bits
      }
      const float f = (float)(1.0 / (sqrt(norm2) + (double)J.eps));
#pragma unroll
      for (int z = 0; z < 8; ++z) {
        const int q = threadIdx.x + z * (32 * kWorkWarps);
        int r, ch;
        if (J.transpose) { ch = q / rows_kept; r = q - ch * rows_kept; }
        else { r = q / cpr; ch = q - r * cpr; }
        if (q >= total) continue;
        uint32_t hi[4], lo[4];
#pragma unroll
        for (int e = 0; e < 4; ++e) split2(u[z][2 * e] * f * kXScale, u[z][2 * e + 1] * f * kXScale, hi[e], lo[e]);
        put_chunk(0, r, ch, hi[0], hi[1], hi[2], hi[3]);
        put_chunk(1, r, ch, lo[0], lo[1], lo[2], lo[3]);
      }
      tc::fence_proxy_async_all();
      __syncwarp();
      if (lane == 0) tc::mbar_arrive(&B->loaded);
      if (!wait(&B->loaded, mat & 1)) break;
      for (int item = sub; item < 8; item += 4) { x_ready(item); partner_ready(item); }

      bool ok = true;
      for (int step = 0; step < J.steps; ++step, ++it) {
        const uint32_t ph = it & 1;
        // ---- A's limbs over its accumulator, and into shared memory
        if (!(ok = wait(&B->m1, ph))) break;
        tc::tc_fence_after_sync();
        uint32_t hi[16], lo[16];
        for (int item = sub; item < a_items; item += 4) {
          if (!works) break;
          uint32_t v[32];
          tc::tmem_ld_32x32(tmem + C::ACC1 + lanes + item * 32, v);
          tc::tmem_ld_wait();
          constexpr float f1 = kAScale / (kXScale * kXScale);
#pragma unroll
          for (int e = 0; e < 16; ++e) split2(__uint_as_float(v[2 * e]) * f1, __uint_as_float(v[2 * e + 1]) * f1, hi[e], lo[e]);
          tc::tmem_st_32x16(tmem + C::ACC1 + lanes + item * 32, hi);
          tc::tmem_st_32x16(tmem + C::ACC1 + lanes + item * 32 + 16, lo);
          const int panel = item >> 1, c0 = (item & 1) * 4;
#pragma unroll
          for (int e = 0; e < 4; ++e)
            tc::st_shared16(sA + panel * kPanel + at_chunk(row, c0 + e), hi[4 * e], hi[4 * e + 1], hi[4 * e + 2], hi[4 * e + 3]);
          if (!PAIR || panel < 2) {
#pragma unroll
            for (int e = 0; e < 4; ++e)
              tc::st_shared16(sA + (C::A_HI + panel) * kPanel + at_chunk(row, c0 + e), lo[4 * e], lo[4 * e + 1], lo[4 * e + 2], lo[4 * e + 3]);
          }
          tc::tmem_st_wait();
          tc::fence_proxy_async_smem();
          tc::tc_fence_before_sync();
          __syncwarp();
          if (lane == 0) arrive(&B->a[panel]);
        }
        if (PAIR) {
          // the low limb's second half, still in registers, follows into the room of the first
          if (!(ok = wait(&B->lofree, ph))) break;
          const int item = sub + 4;
          if (item < a_items) {
#pragma unroll
            for (int e = 0; e < 4; ++e)
              tc::st_shared16(sA + (C::A_HI + (item >> 1) - 2) * kPanel + at_chunk(row, (item & 1) * 4 + e), lo[4 * e], lo[4 * e + 1],
                              lo[4 * e + 2], lo[4 * e + 3]);
            tc::fence_proxy_async_smem();
            __syncwarp();
            if (lane == 0) arrive(&B->l);
          }
        }
        // ---- P = a I + b A + c A A over A's limbs
        if (!(ok = wait(&B->m2, ph))) break;
        tc::tc_fence_after_sync();
        const float fa = J.b * J.p_scale / kAScale, faa = J.cc * J.p_scale / (kAScale * kAScale), fi = J.a * J.p_scale;
        for (int item = sub; item < a_items; item += 4) {
          if (!works) break;
          uint32_t v[32];
          tc::tmem_ld_32x32(tmem + C::ACC2 + lanes + item * 32, v);
          tc::tmem_ld_32x16(tmem + C::ACC1 + lanes + item * 32, hi);
          tc::tmem_ld_32x16(tmem + C::ACC1 + lanes + item * 32 + 16, lo);
          tc::tmem_ld_wait();
#pragma unroll
          for (int e = 0; e < 16; ++e) {
            const float2 h2 = unpack_f16(hi[e]), l2 = unpack_f16(lo[e]);
            float p0 = faa * __uint_as_float(v[2 * e]) + fa * (h2.x + l2.x);
            float p1 = faa * __uint_as_float(v[2 * e + 1]) + fa * (h2.y + l2.y);
            if (grow == item * 32 + 2 * e) p0 += fi;
            if (grow == item * 32 + 2 * e + 1) p1 += fi;
            split2(p0, p1, hi[e], lo[e]);
          }
          tc::tmem_st_32x16(tmem + C::ACC1 + lanes + item * 32, hi);
          tc::tmem_st_32x16(tmem + C::ACC1 + lanes + item * 32 + 16, lo);
          tc::tmem_st_wait();
          tc::tc_fence_before_sync();
          __syncwarp();
          if (lane == 0) arrive(&B->p[item >> 1]);
        }
        // ---- X' over X, or into the weights
        if (!(ok = wait(&B->m3, ph))) break;
        tc::tc_fence_after_sync();
        const bool last = step == J.steps - 1;
        for (int item = sub; item < x_items; item += 4) {
          if (!works) break;
          uint32_t v[32];
          tc::tmem_ld_32x32(tmem + C::ACC3 + lanes + item * 32, v);
          tc::tmem_ld_wait();
          if (!last) {
            const float f3 = 1.0f / J.p_scale;
#pragma unroll
            for (int e = 0; e < 16; ++e) split2(__uint_as_float(v[2 * e]) * f3, __uint_as_float(v[2 * e + 1]) * f3, hi[e], lo[e]);
#pragma unroll
            for (int e = 0; e < 4; ++e) {
              put_chunk(0, row, item * 4 + e, hi[4 * e], hi[4 * e + 1], hi[4 * e + 2], hi[4 * e + 3]);
              put_chunk(1, row, item * 4 + e, lo[4 * e], lo[4 * e + 1], lo[4 * e + 2], lo[4 * e + 3]);
            }
            tc::fence_proxy_async_all();
            tc::tc_fence_before_sync();
            __syncwarp();
            x_ready(item);
            partner_ready(item);
            continue;
          }
          const float fo = 1.0f / (J.p_scale * kXScale);
          const float keep = J.keep, step_w = J.step;
          auto put = [&](int64_t at, float x) {
            if (J.W) J.W[at] = J.W[at] * keep - step_w * x;
            else if (J.o_bf16) static_cast<__nv_bfloat16*>(J.O)[at] = __float2bfloat16_rn(x);
            else static_cast<float*>(J.O)[at] = x;
          };
          if (J.transpose) {                               // lanes are neighbouring columns of W
#pragma unroll
            for (int e = 0; e < 32; ++e) {
              const int j = item * 32 + e;
              if (grow < J.k && j < J.n) put(base + (int64_t)j * J.c + grow, __uint_as_float(v[e]) * fo);
            }
          } else {
            // through this warp's 4 KB of X's room (free now), so that lanes write neighbouring columns
            const uint32_t stage = sX + warp * 4096;
#pragma unroll
            for (int e = 0; e < 32; ++e)
              asm volatile("st.shared.b32 [%0], %1;" ::"r"(stage + (lane * 32 + (e ^ lane)) * 4), "r"(v[e]) : "memory");
            __syncwarp();
            const int j = item * 32 + lane;
#pragma unroll 8
            for (int rr = 0; rr < 32; ++rr) {
              uint32_t x;
              asm volatile("ld.shared.b32 %0, [%1];" : "=r"(x) : "r"(stage + (rr * 32 + (lane ^ rr)) * 4) : "memory");
              const int i = (int)rank * 128 + quarter * 32 + rr;
              if (i < J.k && j < J.n) put(base + (int64_t)i * J.c + j, __uint_as_float(x) * fo);
            }
            __syncwarp();
          }
        }
      }
      tc::tc_fence_before_sync();
      if (!ok) break;
      ++mat;
    }
  }
  if (*abort_flag) {
    if (threadIdx.x == 0) atomicMin(J.status, (int32_t)GNNCO_INTERNAL);
    const long long t0 = clock64();                        // copies and products already issued end before the memory goes
    while (clock64() - t0 < 1000000ll) {}
  }
  tc::tc_fence_before_sync();
  __syncthreads();
  if constexpr (PAIR) {
    tc::cluster_sync_all();
    if (warp == 0) tc::tmem_dealloc_pair(tmem, 512);
  } else {
    if (warp == 0) tc::tmem_dealloc(tmem, 512);
  }
}

template <bool PAIR>
void launch_shape(cudaLaunchConfig_t& cfg, cudaLaunchAttribute* attr, int ctas, cudaStream_t st) {
  cfg.gridDim = dim3(ctas);
  cfg.blockDim = dim3(kThreads);
  cfg.dynamicSmemBytes = Cfg<PAIR>::SMEM;
  cfg.stream = st;
  attr[0].id = cudaLaunchAttributeClusterDimension;
  attr[0].val.clusterDim.x = Cfg<PAIR>::CTAS;
  attr[0].val.clusterDim.y = attr[0].val.clusterDim.z = 1;
  cfg.attrs = attr;
  cfg.numAttrs = 1;
}

// CTA pairs that can be resident at once (asked once per process; 0: none)
int resident_pairs() {
  static const int pairs = [] {
    if (cudaFuncSetAttribute(ns_on_chip<true>, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)Cfg<true>::SMEM) != cudaSuccess) {
      cudaGetLastError();
      return 0;
    }
    cudaLaunchConfig_t cfg{};
    cudaLaunchAttribute attr[1];
    launch_shape<true>(cfg, attr, 2 * 148, nullptr);
    int n = 0;
    if (cudaOccupancyMaxActiveClusters(&n, ns_on_chip<true>, &cfg) != cudaSuccess) {
      cudaGetLastError();
      n = 0;
    }
    return n;
  }();
  return pairs;
}

template <bool PAIR>
int32_t launch(gnnco_handle* h, const NsJob& job, int64_t groups, cudaStream_t st) {
  GNNCO_CUDA_TRY(cudaFuncSetAttribute(ns_on_chip<PAIR>, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)Cfg<PAIR>::SMEM));
  cudaLaunchConfig_t cfg{};
  cudaLaunchAttribute attr[1];
  if (groups > job.sets) groups = job.sets;
  launch_shape<PAIR>(cfg, attr, (int)groups * Cfg<PAIR>::CTAS, st);
  GNNCO_CUDA_TRY(cudaLaunchKernelEx(&cfg, ns_on_chip<PAIR>, job));
  h->launches += 1;
  return GNNCO_OK;
}

}  // namespace

bool ns_on_chip_supported(const gnnco_handle* h, int32_t k, int32_t n) {
  if (k > 256 || n > 256) return false;
  return k <= 128 || resident_pairs() > 0;
}

size_t ns_on_chip_scratch_bytes(const gnnco_handle* h, int64_t sets, int32_t k, int32_t n) {
  if (k <= 128) return 0;
  int64_t pairs = resident_pairs();
  if (pairs > sets) pairs = sets;
  return (size_t)pairs * 8 * kPanel;
}

int32_t launch_ns_on_chip(gnnco_handle* h, const NsJob& job, cudaStream_t st) {
  if (job.k <= 128) return launch<false>(h, job, h->sm_count, st);
  return launch<true>(h, job, resident_pairs(), st);
}
