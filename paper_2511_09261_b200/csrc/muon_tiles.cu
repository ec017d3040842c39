// Newton-Schulz products of matrices that do not fit on one chip area: tiled tensor-core products over the whole GPU, one
// launch per product.
//
//   kGram    A = X X^T                            only tiles (i, j) with j >= i; the mirrored tile is written transposed
//   kPoly    P = a I + b A + c A A                likewise (A is symmetric)
//   kApply   X' = P X, in the last step straight into the weights
//
// Operands are float16 pairs as in muon_tc.cu (hi hi + hi lo + lo hi, float32 accumulators; the small products have an
// accumulator of their own, so that the bits the tensor core drops are small ones).  They live in global scratch (L2) as
// panels of 128 rows x 64 columns, 16 KB, already in the 128-byte-swizzled order of the MMA descriptors: a tile operand
// is one or two contiguous 16-byte-aligned pieces, brought in by untiled bulk copies, and padding to whole panels
// (zeros) leaves no edge cases in the products.  A panel serves as k-major rows and as n-major columns alike.
//
// A tile is 128 x TN (TN = 128, or 64 where tiles are few); a stage of the shared-memory ring holds 64 of k (64 or 48 KB, for 12 MMAs
// of 128 x TN x 16).  k is always summed in four interleaved parts (stages 0, 4, 8 .., then 1, 5, 9 ..), added in that order:
// one CTA takes the parts in turn, in two accumulator buffers; with few tiles and a long k a cluster of four CTAs takes one
// part each, hands the others their column group of its partial tile through distributed shared memory, and finishes its
// own group.  The results are the same bits in all forms.  (The exchange takes 4.7 us, as long as nine stages: clusters pay
// from some 40 stages on, below that narrow tiles spread the work better.)
// 1,000 x 1,537 takes 243 us: 15 products of 13 to 15 us (0.5 us a stage, near the 0.4 us of its MMAs), each with 2 us until the next one
// starts, 1 us until its first operands arrive and 2 to 3 us of conversion and stores.
// Launches are chained by programmatic dependence: a kernel sets itself up while the one before it finishes.
// Roles: warps 0-7 epilogue (TMEM lanes 32 (w % 4), column half w / 4), warp 8 issues MMAs, warp 9 the copies.
#include <cuda_fp16.h>
#include <math.h>

#include "muon_internal.cuh"
#include "muon_limbs.cuh"
#include "tc_common.cuh"
#include "vec_io.cuh"
#include "walk.cuh"

namespace {

constexpr int kGram = 0, kPoly = 1, kApply = 2;
constexpr int kEpiWarps = 8, kMmaWarp = 8, kCopyWarp = 9, kThreads = 320;
constexpr uint32_t kRing = 12 * kPanel;                    // 3 stages of 64 KB or 4 of 48 KB
constexpr size_t kSmem = 1024 + kRing + 256;

struct TileJob {
  const uint8_t *left, *right, *mid;                       // limbs: left and right operand, A where P is formed
  uint8_t* out;
  int64_t left_set, right_set, out_set;                    // bytes between matrices
  uint32_t left_limb, right_limb, out_limb;                // bytes between limbs
  int32_t rb;                                              // row tiles (128) of X, A and P
  int32_t cb;                                              // 64-column panels of X (an even number)
  int32_t stages;                                          // 64-wide steps of the contraction
  int32_t last;
  NsJob J;
  int64_t set0;
};

__device__ __forceinline__ bool wait_bounded(uint64_t* bar, uint32_t parity, volatile uint32_t* abort_flag) {
  if (tc::mbar_try_wait(bar, parity)) return true;
  const long long t0 = clock64();
  while (!tc::mbar_try_wait(bar, parity)) {
    if (*abort_flag) return false;
    if (clock64() - t0 > 4000000000ll) {
      *abort_flag = 1;
      return false;
    }
  }
  return true;
}

// upper-triangular tile number -> (i, j), j >= i
__device__ __forceinline__ void tile_of(int t, int n, int& i, int& j) {
  i = 0;
  while (t >= n - i) {
    t -= n - i;
    ++i;
  }
  j = i + t;
}

template <int KIND, int TN, int SPLIT>
__global__ void __launch_bounds__(kThreads, 1) ns_tiles(const TileJob T) {
  static_assert(SPLIT == 1 || (KIND == kGram && TN == 128), "clusters take tiles of X X^T");
  constexpr uint32_t kStageBytes = 2 * kPanel + 2 * TN * 128;
  constexpr int kStages = kRing / kStageBytes;
  constexpr uint32_t B_LIMB = TN * 128;                    // bytes of the right operand's limb in a stage

  const NsJob& J = T.J;
  const int64_t s = blockIdx.y;
  asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
  if (J.active && !J.active[T.set0 + s]) return;           // the whole cluster leaves
  extern __shared__ uint8_t smem_raw[];
  const uint32_t sbase = (tc::smem_u32(smem_raw) + 1023u) & ~1023u;
  uint8_t* gen = smem_raw + (sbase - tc::smem_u32(smem_raw));
  uint64_t* full = reinterpret_cast<uint64_t*>(gen + kRing);
  uint64_t* empty = full + kStages;
  uint64_t* done = empty + kStages;                         // [4] a part's products are complete
  uint64_t* freed = done + 4;                              // [2] its accumulators have been read
  uint32_t* tmem_slot = reinterpret_cast<uint32_t*>(freed + 2);
  volatile uint32_t* abort_flag = tmem_slot + 1;
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const uint32_t rank = SPLIT > 1 ? tc::cluster_ctarank() : 0u;
  const int tile = blockIdx.x / SPLIT;
  int ti, tj;                                              // row tile, column tile of TN columns
  if (KIND == kApply) {
    ti = tile % T.rb;
    tj = tile / T.rb;
  } else if (TN == 128) {
    tile_of(tile, T.rb, ti, tj);
  } else {
    tile_of(tile >> 1, T.rb, ti, tj);
    tj = 2 * tj + (tile & 1);
  }
  const int tr = TN == 128 ? tj : tj >> 1;                 // row tile of the right operand of A A and X X^T,
  const uint32_t tr_off = TN == 128 ? 0u : (uint32_t)(tj & 1) * (kPanel / 2);   // and the tile's 64 rows in it
  const bool same = KIND != kApply && ti == tr;            // a diagonal tile: the left operand's rows are the right one's
  constexpr int kParts = 4 / SPLIT;                        // parts this CTA sums: first, first + 1 ..
  const int first = (int)rank * kParts;
  auto part_stages = [&](int p) { return (T.stages - (first + p) + 3) / 4; };

  if (threadIdx.x == 0) {
    for (int i = 0; i < kStages; ++i) {
      tc::mbar_init(full + i, 1);
      tc::mbar_init(empty + i, 1);
    }
    for (int i = 0; i < 4; ++i) tc::mbar_init(done + i, 1);
    for (int i = 0; i < 2; ++i) tc::mbar_init(freed + i, kEpiWarps);
    *abort_flag = 0;
    tc::fence_mbar_init();
  }
  constexpr uint32_t kCols = (kParts > 1 ? 4 : 2) * TN;
  if (warp == 0) tc::tmem_alloc(tmem_slot, kCols);
  tc::tc_fence_before_sync();
  __syncthreads();
  tc::tc_fence_after_sync();
  const uint32_t tmem = *tmem_slot;
  asm volatile("griddepcontrol.wait;" ::: "memory");       // the operands of this product are complete from here on

  if (warp == kCopyWarp) {
    if (lane == 0) {
      const uint8_t* lp = T.left + s * T.left_set;
      const uint8_t* rp = T.right + s * T.right_set;
      int q = 0;
      bool ok = true;
      for (int p = 0; p < kParts && ok; ++p)
      for (int kb = first + p; kb < T.stages; kb += 4, ++q) {
        const int slot = q % kStages, use = q / kStages;
        if (use > 0 && !(ok = wait_bounded(empty + slot, (use - 1) & 1, abort_flag))) break;
        const uint32_t at = sbase + slot * kStageBytes;
        tc::mbar_arrive_expect_tx(full + slot, same ? 2 * kPanel : kStageBytes);
        for (int limb = 0; limb < 2; ++limb) {
          tc::bulk_load(at + limb * kPanel, lp + limb * (int64_t)T.left_limb + ((int64_t)kb * T.rb + ti) * kPanel, kPanel, full + slot);
          if (same) continue;
          const uint32_t to = at + 2 * kPanel + limb * B_LIMB;
          const uint8_t* const from = rp + limb * (int64_t)T.right_limb;
          if (KIND != kApply) {
            tc::bulk_load(to, from + ((int64_t)kb * T.rb + tr) * kPanel + tr_off, B_LIMB, full + slot);
          } else {
            // 64 rows of the tile's panels of X
            for (int h = 0; h < TN / 64; ++h)
              tc::bulk_load(to + h * (kPanel / 2), from + ((int64_t)(tj * (TN / 64) + h) * T.rb + (kb >> 1)) * kPanel + (kb & 1) * (kPanel / 2),
                            kPanel / 2, full + slot);
          }
        }
      }
    }
    __syncwarp();
    if (KIND == kApply && T.last && J.W) {
      // the tile of W that the products are about to be added to
      const int64_t base = (T.set0 + s) * (int64_t)J.r * J.c;
      const int row0 = J.transpose ? tj * TN : ti * 128, col0 = J.transpose ? ti * 128 : tj * TN;
      const int tile_rows = J.transpose ? TN : 128, tile_cols = J.transpose ? 128 : TN;
      for (int q = lane; q < tile_rows * 5; q += 32) {
        const int i = row0 + q / 5, j = min(col0 + (q % 5) * 32, min(col0 + tile_cols - 1, J.c - 1));
        if (i < J.r) asm volatile("prefetch.global.L2 [%0];" ::"l"(J.W + base + (int64_t)i * J.c + j));
      }
    }
  } else if (warp == kMmaWarp) {
    const uint32_t leader = tc::elect_one();
    const uint32_t idesc = tc::idesc_f16_f32(128, TN, KIND == kApply);
    const uint32_t tb = __shfl_sync(0xffffffffu, tmem, 0);
    bool ok = true;
    int q = 0;
    for (int p = 0; p < kParts && ok; ++p) {
      const int count = part_stages(p);
      const uint32_t big = tb + (p & 1) * (2 * TN), small = big + TN;
      // buffers are reused by parts 2 and 3; an empty part neither completes nor frees anything
      if (p >= 2 && count > 0) ok = __all_sync(0xffffffffu, wait_bounded(freed + (p & 1), 0, abort_flag)) != 0;
      tc::tc_fence_after_sync();
      for (int g = 0; g < count && ok; ++g, ++q) {
        const int slot = q % kStages, use = q / kStages;
        ok = __all_sync(0xffffffffu, wait_bounded(full + slot, use & 1, abort_flag)) != 0;
        tc::tc_fence_after_sync();
        if (!ok) break;
        const uint32_t at = sbase + slot * kStageBytes;
        const uint64_t ah = tc::smem_desc_sw128(at, 16, 1024), al = tc::smem_desc_sw128(at + kPanel, 16, 1024);
        const uint32_t bt = at + (same ? tr_off : 2 * kPanel), b_limb = same ? kPanel : B_LIMB;
        const uint32_t lbo = KIND == kApply ? kPanel / 2 : 16;
        const uint64_t bh = tc::smem_desc_sw128(bt, lbo, 1024), bl = tc::smem_desc_sw128(bt + b_limb, lbo, 1024);
        constexpr uint64_t bstep = KIND == kApply ? 128 : 2; // 16 of k: 2,048 bytes of n-major rows, 32 of k-major ones
#pragma unroll
        for (int k = 0; k < 4; ++k) {
          tc::mma_f16<false, false>(leader, big, ah + 2 * k, bh + bstep * k, idesc, g + k != 0);
          tc::mma_f16<false, false>(leader, small, ah + 2 * k, bl + bstep * k, idesc, g + k != 0);
          tc::mma_f16<false, false>(leader, small, al + 2 * k, bh + bstep * k, idesc, true);
        }
        if (leader) tc::mma_commit(empty + slot);
        __syncwarp();
      }
      if (ok && leader && count > 0) tc::mma_commit(done + p);
      __syncwarp();
    }
  }
  // ---- partial tiles to registers: items (32 columns) half and, in wide tiles, half + 2; the parts in order
  const int quarter = warp & 3, half = warp >> 2;          // of the epilogue warps
  const int row = quarter * 32 + lane;
  const uint32_t lanes = (uint32_t)(quarter * 32) << 16;
  constexpr int NI = TN / 64;                              // items of a warp
  float sum[NI][32];
  if (warp < kEpiWarps) {
#pragma unroll
    for (int i = 0; i < NI; ++i)
#pragma unroll
      for (int e = 0; e < 32; ++e) sum[i][e] = 0.0f;
    for (int p = 0; p < kParts; ++p) {
      if (part_stages(p) <= 0) continue;
      if (!wait_bounded(done + p, 0, abort_flag)) break;
      tc::tc_fence_after_sync();
#pragma unroll
      for (int i = 0; i < NI; ++i) {
        uint32_t v[32], w[32];
        const uint32_t at = tmem + (p & 1) * (2 * TN) + lanes + (half + 2 * i) * 32;
        tc::tmem_ld_32x32(at, v);
        tc::tmem_ld_32x32(at + TN, w);
        tc::tmem_ld_wait();
#pragma unroll
        for (int e = 0; e < 32; ++e) sum[i][e] += __uint_as_float(v[e]) + __uint_as_float(w[e]);
      }
      tc::tc_fence_before_sync();
      __syncwarp();
      if (kParts > 1 && p < 2 && lane == 0) tc::mbar_arrive(freed + p);
    }
  }
  tc::tc_fence_before_sync();
  __syncthreads();                                         // the ring is free: every copy has been consumed
  tc::tc_fence_after_sync();

  if constexpr (SPLIT > 1) {
    // partial tiles to their owners: [from CTA][row][32 columns], 16 KB each
    tc::cluster_sync_all();                                // every CTA's ring is free
    if (warp < kEpiWarps) {
#pragma unroll
      for (int i = 0; i < NI; ++i) {
        const uint32_t to = tc::map_to_cta(sbase + rank * kPanel, half + 2 * i);
#pragma unroll
        for (int e = 0; e < 8; ++e)
          asm volatile("st.shared::cluster.v4.f32 [%0], {%1, %2, %3, %4};" ::"r"(to + at_chunk(row, e)), "f"(sum[i][4 * e]), "f"(sum[i][4 * e + 1]),
                       "f"(sum[i][4 * e + 2]), "f"(sum[i][4 * e + 3]) : "memory");
      }
    }
    tc::cluster_sync_all();
  }
  if (warp < kEpiWarps && !*abort_flag) {
    // one CTA: this warp's items; a cluster: the CTA's own one, by its first four warps
#pragma unroll
    for (int i = 0; i < NI; ++i) {
      if (SPLIT > 1 && (half > 0 || i > 0)) continue;
      const int item = SPLIT > 1 ? (int)rank : half + 2 * i;
      uint32_t v[32];
      if constexpr (SPLIT > 1) {
        float total[32];
#pragma unroll
        for (int e = 0; e < 32; ++e) total[e] = 0.0f;
        for (int from = 0; from < SPLIT; ++from)
#pragma unroll
          for (int e = 0; e < 8; ++e) {
            const uint4 a = tc::ld_shared16(sbase + from * kPanel + at_chunk(row, e));
            total[4 * e] += __uint_as_float(a.x);
            total[4 * e + 1] += __uint_as_float(a.y);
            total[4 * e + 2] += __uint_as_float(a.z);
            total[4 * e + 3] += __uint_as_float(a.w);
          }
#pragma unroll
        for (int e = 0; e < 32; ++e) v[e] = __float_as_uint(total[e]);
      } else {
#pragma unroll
        for (int e = 0; e < 32; ++e) v[e] = __float_as_uint(sum[i][e]);
      }
      const int c0 = item * 32;                            // first column inside the tile
      const int panel = (TN / 64) * tj + (c0 >> 6), chunk0 = (c0 & 63) >> 3;
      uint8_t* const to = T.out + s * T.out_set + ((int64_t)panel * T.rb + ti) * kPanel;
      if (KIND == kApply && T.last) {
        const float fo = 1.0f / (J.p_scale * kXScale);
        const int64_t base = (T.set0 + s) * (int64_t)J.r * J.c;
        auto put = [&](int64_t at, float w, float x) {
          if (J.W) __stcs(J.W + at, w * J.keep - J.step * x);
          else if (J.o_bf16) static_cast<__nv_bfloat16*>(J.O)[at] = __float2bfloat16_rn(x);
          else __stcs(static_cast<float*>(J.O) + at, x);
        };
        if (J.transpose) {                                 // lanes are neighbouring columns of W
          const int i = ti * 128 + row, j0 = tj * TN + c0;
          float w[32];
#pragma unroll
          for (int e = 0; e < 32; ++e) w[e] = J.W && i < J.k && j0 + e < J.n ? __ldcs(J.W + base + (int64_t)(j0 + e) * J.c + i) : 0.0f;
#pragma unroll
          for (int e = 0; e < 32; ++e)
            if (i < J.k && j0 + e < J.n) put(base + (int64_t)(j0 + e) * J.c + i, w[e], __uint_as_float(v[e]) * fo);
        } else {
          // rows pass through shared memory, so that lanes work on neighbouring columns
          const uint32_t stage = sbase + warp * 4096;
#pragma unroll
          for (int e = 0; e < 8; ++e) tc::st_shared16(stage + at_chunk(lane, e), v[4 * e], v[4 * e + 1], v[4 * e + 2], v[4 * e + 3]);
          __syncwarp();
          const int j = tj * TN + c0 + lane;
          float w[32];
#pragma unroll
          for (int e = 0; e < 32; ++e) {
            const int i = ti * 128 + quarter * 32 + e;
            w[e] = J.W && i < J.k && j < J.n ? __ldcs(J.W + base + (int64_t)i * J.c + j) : 0.0f;
          }
#pragma unroll
          for (int e = 0; e < 32; ++e) {
            uint32_t x;
            asm volatile("ld.shared.b32 %0, [%1];" : "=r"(x) : "r"(stage + at_chunk(e, lane >> 2) + (lane & 3) * 4) : "memory");
            const int i = ti * 128 + quarter * 32 + e;
            if (i < J.k && j < J.n) put(base + (int64_t)i * J.c + j, w[e], __uint_as_float(x) * fo);
          }
          __syncwarp();
        }
        continue;
      }
      uint32_t hi[16], lo[16];
      if (KIND == kPoly) {
        const uint8_t* const am = T.mid + s * T.left_set + ((int64_t)panel * T.rb + ti) * kPanel;
        const float fi = J.a * J.p_scale, fa = J.b * J.p_scale / kAScale, faa = J.cc * J.p_scale / (kAScale * kAScale);
        // (plain loads: this kernel may have been running while A was written, which rules the read-only path out.  Two chunks of a
        // row share a 32-byte sector, so the loads stay cacheable in L1: past it 120 x 260 x 300 took 1,125 us instead of 1,091.)
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          const uint4 h4 = *reinterpret_cast<const uint4*>(am + at_chunk(row, chunk0 + e));
          const uint4 l4 = *reinterpret_cast<const uint4*>(am + T.left_limb + at_chunk(row, chunk0 + e));
          hi[4 * e] = h4.x; hi[4 * e + 1] = h4.y; hi[4 * e + 2] = h4.z; hi[4 * e + 3] = h4.w;
          lo[4 * e] = l4.x; lo[4 * e + 1] = l4.y; lo[4 * e + 2] = l4.z; lo[4 * e + 3] = l4.w;
        }
        const int diag = ti * 128 + row - (tj * TN + c0);  // this row's place on the diagonal, if it is in the item
#pragma unroll
        for (int e = 0; e < 16; ++e) {
          const float2 A2 = join2(hi[e], lo[e]);
          v[2 * e] = __float_as_uint(fmaf(fa, A2.x, faa * __uint_as_float(v[2 * e])) + (diag == 2 * e ? fi : 0.0f));
          v[2 * e + 1] = __float_as_uint(fmaf(fa, A2.y, faa * __uint_as_float(v[2 * e + 1])) + (diag == 2 * e + 1 ? fi : 0.0f));
        }
      }
      const float f1 = KIND == kGram ? kAScale / (kXScale * kXScale) : KIND == kPoly ? 1.0f : 1.0f / J.p_scale;
      const uint64_t f = pair_of(f1, f1);
#pragma unroll
      for (int e = 0; e < 16; ++e) split2_scaled(v[2 * e], v[2 * e + 1], f, hi[e], lo[e]);
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        *reinterpret_cast<uint4*>(to + at_chunk(row, chunk0 + e)) = make_uint4(hi[4 * e], hi[4 * e + 1], hi[4 * e + 2], hi[4 * e + 3]);
        *reinterpret_cast<uint4*>(to + T.out_limb + at_chunk(row, chunk0 + e)) = make_uint4(lo[4 * e], lo[4 * e + 1], lo[4 * e + 2], lo[4 * e + 3]);
      }
      if (KIND != kApply && !same) {
        // the mirrored tile: row tr_row + e of row tile tr, column `row` (lanes write neighbouring float16 values)
        uint8_t* const mt = T.out + s * T.out_set + ((int64_t)(2 * ti + (row >> 6)) * T.rb + tr) * kPanel;
        const int cc = (row & 63) >> 3, tr_row = (int)(tr_off >> 7) + c0;
#pragma unroll
        for (int e = 0; e < 32; ++e) {
          const uint32_t o = at_chunk(tr_row + e, cc) + (row & 7) * 2;
          *reinterpret_cast<unsigned short*>(mt + o) = (unsigned short)(e & 1 ? hi[e >> 1] >> 16 : hi[e >> 1] & 0xffffu);
          *reinterpret_cast<unsigned short*>(mt + T.out_limb + o) = (unsigned short)(e & 1 ? lo[e >> 1] >> 16 : lo[e >> 1] & 0xffffu);
        }
      }
    }
  }
  if (*abort_flag) {
    if (threadIdx.x == 0) atomicMin(J.status, (int32_t)GNNCO_INTERNAL);
    const long long t0 = clock64();                        // copies and products already issued end before the memory goes
    while (clock64() - t0 < 1000000ll) {}
  }
  tc::tc_fence_before_sync();
  __syncthreads();
  if (warp == 0) tc::tmem_dealloc(tmem, kCols);
}

// u from the gradient (and the updated momentum), scaled, as limbs in panels: one thread per 8 columns of a row of X
template <typename TG>
__global__ void __launch_bounds__(256) ns_pack(const NsJob J, int64_t set0, const double* __restrict__ partial, int parts, uint8_t* __restrict__ X,
                                               int64_t x_set, uint32_t x_limb, int32_t rb, int32_t cb) {
  const int64_t s = blockIdx.y;
  if (J.active && !J.active[set0 + s]) return;
  // every block adds the same partial sums in the same order (at most 256, one per thread)
  __shared__ double part_sum[8];
  double t = (int)threadIdx.x < parts ? partial[s * parts + threadIdx.x] : 0.0;
#pragma unroll
  for (int d = 16; d > 0; d >>= 1) t += __shfl_xor_sync(0xffffffffu, t, d);
  if ((threadIdx.x & 31) == 0) part_sum[threadIdx.x >> 5] = t;
  __syncthreads();
  t = 0.0;
#pragma unroll
  for (int w = 0; w < 8; ++w) t += part_sum[w];
  const NsFactor by = ns_factor(t, J.eps, kXScale);
  const int rows = rb * 128, chunks = cb * 8;
  const int64_t base = (set0 + s) * (int64_t)J.r * J.c;
  for (int64_t q = (int64_t)blockIdx.x * 256 + threadIdx.x; q < (int64_t)rows * chunks; q += (int64_t)gridDim.x * 256) {
    // lanes along whichever index is contiguous in memory
    const int i = J.transpose ? (int)(q % rows) : (int)(q / chunks), ch = J.transpose ? (int)(q / rows) : (int)(q % chunks);
    uint32_t hi[4], lo[4];
    float u[8];
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      const int j = ch * 8 + e;
      u[e] = 0.0f;
      if (i < J.k && j < J.n) {
        const int64_t at = base + (J.transpose ? (int64_t)j * J.c + i : (int64_t)i * J.c + j);
        vio::Raw<TG, 1> g;
        g.template load<false>(static_cast<const TG*>(J.G) + at);
        u[e] = J.m ? (J.nesterov ? g.get(0) + J.mu * J.m[at] : J.m[at]) : g.get(0);
      }
    }
#pragma unroll
    for (int e = 0; e < 4; ++e) split2(u[2 * e] * by.lift * by.f, u[2 * e + 1] * by.lift * by.f, hi[e], lo[e]);
    uint8_t* const to = X + s * x_set + ((int64_t)(ch >> 3) * rb + (i >> 7)) * kPanel + at_chunk(i & 127, ch & 7);
    *reinterpret_cast<uint4*>(to) = make_uint4(hi[0], hi[1], hi[2], hi[3]);
    *reinterpret_cast<uint4*>(to + x_limb) = make_uint4(lo[0], lo[1], lo[2], lo[3]);
  }
}

// momentum in place and the sum of squares of u: grid (blocks, sets), one float64 partial sum per block
template <typename TG>
__global__ void __launch_bounds__(256) ns_momentum(const NsJob J, int64_t set0, double* __restrict__ partial) {
  const int64_t s = blockIdx.y, base = (set0 + s) * (int64_t)J.r * J.c;
  if (J.active && !J.active[set0 + s]) return;
  const int64_t count = (int64_t)J.r * J.c;
  double sum = 0.0;
  for (PieceWalk piece(count, blockIdx.x, gridDim.x, 1024); piece.more(); piece.next()) {
    vio::Raw<TG, 1> g[4];
    float mv[4];
#pragma unroll
    for (int y = 0; y < 4; ++y) {
      const int64_t q = piece.at + y * 256 + (int)threadIdx.x;
      g[y].zero();
      mv[y] = 0.0f;
      if (q < count) {
        g[y].template load<true>(static_cast<const TG*>(J.G) + base + q);
        if (J.m) mv[y] = J.m[base + q];
      }
    }
#pragma unroll
    for (int y = 0; y < 4; ++y) {
      const int64_t q = piece.at + y * 256 + (int)threadIdx.x;
      if (q >= count) continue;
      float u = g[y].get(0);
      if (J.m) {
        const float v = J.mu * mv[y] + u;
        J.m[base + q] = v;
        u = J.nesterov ? u + J.mu * v : v;
      }
      sum += (double)u * (double)u;
    }
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

constexpr int kMaxParts = 256;                             // partial sums of squares per matrix
int parts_of(int64_t count) {
  const int64_t p = (count + 8191) / 8192;
  return (int)(p < 1 ? 1 : p > kMaxParts ? kMaxParts : p);
}

struct Layout {
  uint8_t *x0, *x1, *a, *p;
  double* partial;
  int64_t x_set, a_set, chunk;                             // bytes per matrix; matrices worked on at a time
  uint32_t x_limb, a_limb;
  int32_t rb, cb;
  size_t bytes;
};
Layout layout(void* ws, int64_t sets, int32_t k, int32_t n) {
  Layout L;
  L.rb = (k + 127) / 128;
  L.cb = (n + 127) / 128 * 2;
  L.x_limb = (uint32_t)L.cb * L.rb * kPanel;
  L.a_limb = (uint32_t)2 * L.rb * L.rb * kPanel;
  L.x_set = 2 * (int64_t)L.x_limb;
  L.a_set = 2 * (int64_t)L.a_limb;
  // at least four tiles per SM, so that a chunk's launches fill the GPU; beyond that L2 is better kept small
  const int64_t tiles = (int64_t)L.rb * (L.rb + 1) / 2;
  L.chunk = (148 * 4 + tiles - 1) / tiles;
  if (L.chunk > sets) L.chunk = sets;
  Carver c(ws, 0);
  L.x0 = c.take<uint8_t>(L.chunk * L.x_set);
  L.x1 = c.take<uint8_t>(L.chunk * L.x_set);
  L.a = c.take<uint8_t>(L.chunk * L.a_set);
  L.p = c.take<uint8_t>(L.chunk * L.a_set);
  L.partial = c.take<double>(L.chunk * kMaxParts);
  L.bytes = c.off;
  return L;
}

template <int KIND, int TN, int SPLIT>
int32_t launch_form(gnnco_handle* h, const TileJob& T, int64_t tiles, unsigned sets, cudaStream_t st) {
  auto kernel = ns_tiles<KIND, TN, SPLIT>;
  static std::atomic<int> allowed{0};
  const int32_t rc = allow_shared_memory(kernel, kSmem, h->device, allowed);
  if (rc != GNNCO_OK) return rc;
  cudaLaunchConfig_t cfg{};
  cfg.gridDim = dim3((unsigned)(tiles * SPLIT), sets);
  cfg.blockDim = dim3(kThreads);
  cfg.dynamicSmemBytes = kSmem;
  cfg.stream = st;
  cudaLaunchAttribute attr[2];
  attr[0].id = cudaLaunchAttributeClusterDimension;
  attr[0].val.clusterDim.x = SPLIT;
  attr[0].val.clusterDim.y = attr[0].val.clusterDim.z = 1;
  attr[1].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr[1].val.programmaticStreamSerializationAllowed = 1;
  cfg.attrs = attr;
  cfg.numAttrs = 2;
  GNNCO_CUDA_TRY(cudaLaunchKernelEx(&cfg, kernel, T));
  h->launches += 1;
  return GNNCO_OK;
}

// Clusters of four that can be resident at once (asked once per process): fewer than SMs / 4, since a cluster stays inside one
// group of SMs.
int resident_quads() {
  static const int quads = [] {
    auto kernel = ns_tiles<kGram, 128, 4>;
    if (cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)kSmem) != cudaSuccess) {
      cudaGetLastError();
      return 0;
    }
    cudaLaunchConfig_t cfg{};
    cfg.gridDim = dim3(4 * 37);
    cfg.blockDim = dim3(kThreads);
    cfg.dynamicSmemBytes = kSmem;
    cudaLaunchAttribute attr[1];
    attr[0].id = cudaLaunchAttributeClusterDimension;
    attr[0].val.clusterDim.x = 4;
    attr[0].val.clusterDim.y = attr[0].val.clusterDim.z = 1;
    cfg.attrs = attr;
    cfg.numAttrs = 1;
    int n = 0;
    if (cudaOccupancyMaxActiveClusters(&n, kernel, &cfg) != cudaSuccess) {
      cudaGetLastError();
      n = 0;
    }
    return n;
  }();
  return quads;
}

// `tiles` counts tiles of 128 columns.  Narrow tiles while they leave SMs free; a cluster per tile for a long k, where the GPU holds
// them all at once.  (A long k of A A or P X is a long side of A, whose tiles are too many for that: X X^T only.)
constexpr int kLongStages = 40;
template <int KIND>
int32_t launch_product(gnnco_handle* h, const TileJob& T, int64_t tiles, unsigned sets, cudaStream_t st) {
  if constexpr (KIND == kGram)
    if (T.stages >= kLongStages && tiles * sets <= resident_quads()) return launch_form<KIND, 128, 4>(h, T, tiles, sets, st);
  if (tiles * sets * 2 <= h->sm_count) return launch_form<KIND, 64, 1>(h, T, 2 * tiles, sets, st);
  return launch_form<KIND, 128, 1>(h, T, tiles, sets, st);
}

template <typename TG>
int32_t run(gnnco_handle* h, const NsJob& J, const Layout& L, cudaStream_t st) {
  const int parts = parts_of((int64_t)J.r * J.c);
  for (int64_t s0 = 0; s0 < J.sets; s0 += L.chunk) {
    const unsigned ns = (unsigned)(J.sets - s0 < L.chunk ? J.sets - s0 : L.chunk);
    ns_momentum<TG><<<dim3(parts, ns), 256, 0, st>>>(J, s0, L.partial);
    const int64_t units = (int64_t)L.rb * 128 * L.cb * 8;
    const int64_t pb = (units + 255) / 256;
    ns_pack<TG><<<dim3((unsigned)(pb < 1024 ? pb : 1024), ns), 256, 0, st>>>(J, s0, L.partial, parts, L.x0, L.x_set, L.x_limb, L.rb, L.cb);
    h->launches += 2;
    GNNCO_LAUNCH_CHECK();
    uint8_t *x = L.x0, *y = L.x1;
    const int64_t sym = (int64_t)L.rb * (L.rb + 1) / 2;
    for (int t = 0; t < J.steps; ++t) {
      TileJob T = {};
      T.J = J;
      T.set0 = s0;
      T.rb = L.rb;
      T.cb = L.cb;
      T.left = T.right = x; T.left_set = T.right_set = L.x_set; T.left_limb = T.right_limb = L.x_limb;
      T.out = L.a; T.out_set = L.a_set; T.out_limb = L.a_limb;
      T.stages = (J.n + 63) / 64;
      int32_t rc = launch_product<kGram>(h, T, sym, ns, st);
      if (rc != GNNCO_OK) return rc;
      T.left = T.right = T.mid = L.a; T.left_set = T.right_set = L.a_set; T.left_limb = T.right_limb = L.a_limb;
      T.out = L.p;
      T.stages = (J.k + 63) / 64;
      if ((rc = launch_product<kPoly>(h, T, sym, ns, st)) != GNNCO_OK) return rc;
      T.left = L.p; T.right = x; T.right_set = L.x_set; T.right_limb = L.x_limb;
      T.out = y; T.out_set = L.x_set; T.out_limb = L.x_limb;
      T.last = t == J.steps - 1;
      if ((rc = launch_product<kApply>(h, T, (int64_t)L.rb * (L.cb / 2), ns, st)) != GNNCO_OK) return rc;
      uint8_t* q = x; x = y; y = q;
    }
  }
  return GNNCO_OK;
}

}  // namespace

bool ns_tiles_supported(int32_t k, int32_t n) {
  // limb strides are 32-bit
  return (int64_t)((k + 127) / 128) * ((n + 127) / 128) * 2 * kPanel < ((int64_t)1 << 32);
}
size_t ns_tiles_workspace_bytes(int64_t sets, int32_t k, int32_t n) { return layout(nullptr, sets, k, n).bytes; }
int32_t launch_ns_tiles(gnnco_handle* h, const NsJob& job, void* ws, cudaStream_t st) {
  const Layout L = layout(ws, job.sets, job.k, job.n);
  return job.g_bf16 ? run<__nv_bfloat16>(h, job, L, st) : run<float>(h, job, L, st);
}
