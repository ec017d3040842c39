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
// times (error of a 256 x 256 iterate after 5 steps: 3.8e-6, 8.0e-6 when interleaved).  That is float32 accuracy at a
// third of the float16 rate; one float16 or bfloat16 product would put 2e-3 (1.5e-2) into the result, because errors
// in the direction of small singular values grow by a = 3.4 per step.
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
// What bounds it.  4,096 x 256 x 256 (6.2 PFLOP of float16 products, three per float32 one): 6.3 ms, the power cap
// holding the clock at 1.7 GHz (592 x 256 x 256, too short for that: 861 us); the tensor pipe is active half of the time.
// A step of a pair takes 27,700 cycles, 18,400 of them products: what is left are the conversions between them that
// nothing covers.  Loading and storing a matrix takes 48,000 cycles; starting the pairs at different times did not
// change that.  1,024 x 128 x 128: 251 us (235 where the same matrices are updated again and again, as far as they stay in L2).
//
// Roles: after the working warps (16; 8 where two CTAs share an SM) one warp issues MMAs, and in a pair another
// exchanges blocks; the working warps load, convert and store: warp w owns rows 32 (w % 4) .. +32 (its TMEM lanes) and
// the 32-column items w / 4 and w / 4 + 4.  Barriers per 64-column panel let the next product start on the first panels
// while the others are converted.  Every wait is bounded; a CTA that gives up raises the status word.
#include <cuda_fp16.h>
#include <math.h>

#include <type_traits>

#include "muon_internal.cuh"
#include "muon_limbs.cuh"
#include "tc_common.cuh"
#include "vec_io.cuh"

namespace {

// kDual: both sides up to 128, two CTAs per SM (while one converts, the other's products run: 1,024 x 128 x 128 took
// 272 us so and 334 with one when this was decided); kWide: short side up to 128, long side up to 256, one CTA per SM;
// kPair: sides up to 256, two CTAs on two SMs.
constexpr int kDual = 0, kWide = 1, kPair = 2;

template <int MODE>
struct Cfg {
  static constexpr bool PAIR = MODE == kPair;
  static constexpr int CTAS = PAIR ? 2 : 1, PER_SM = MODE == kDual ? 2 : 1;
  static constexpr int WORK = MODE == kDual ? 8 : 16;      // working warps; then the MMA warp and, in a pair, the side warp
  static constexpr int SUBS = WORK / 4, THREADS = 32 * (WORK + 1 + (PAIR ? 1 : 0));
  static constexpr int XP = MODE == kDual ? 2 : 4;         // panels of X per limb
  static constexpr int A_HI = PAIR ? 4 : 2, A_LO = MODE == kDual ? 1 : 2;   // panels of A's limbs in shared memory
  static constexpr bool LATE = A_LO < A_HI;                // the low limb's second half follows into the room of the first
  static constexpr uint32_t X_BYTES = 2 * XP * kPanel, A_BYTES = (A_HI + A_LO) * kPanel, MISC = 1024;
  // two CTAs fill an SM's shared memory to the byte: no slack for aligning the base, which starts on 1,024 bytes
  static constexpr uint32_t SLACK = MODE == kDual ? 0 : 1024;
  static constexpr size_t SMEM = SLACK + X_BYTES + A_BYTES + MISC;
  static constexpr uint32_t ACC1 = 0, ACC2 = PAIR ? 256 : 128, ACC3 = MODE == kDual ? 128 : 256;   // TMEM columns
  static constexpr bool SHARED_ACC = ACC2 == ACC3;
  static constexpr uint32_t TMEM = MODE == kDual ? 256 : 512;
  static_assert(SMEM <= 232448 && PER_SM * (SMEM + 1024) <= 233472, "does not fit in shared memory");
};

struct Bars {
  uint64_t x[4], a[4], p[4];                               // panel ready (used in the even CTA)
  uint64_t m1, m2, m3, lofree;                             // products done (both CTAs)
  uint64_t l;                                              // second half of A's low limb ready (even CTA)
  uint64_t own;                                            // this CTA's off-diagonal block written (by its workers)
  uint64_t g, s, s2;                                       // partner's block in scratch / copied here / copied there
  uint64_t norm, again, loaded;                            // loader: sums ready, sums read, X written
  uint64_t peer1, peer2;                                   // partner's sum of the first / second round ready
};

__device__ __forceinline__ void st_shared8(uint32_t saddr, uint32_t a, uint32_t b) {
  asm volatile("st.shared.v2.u32 [%0], {%1, %2};" ::"r"(saddr), "r"(a), "r"(b) : "memory");
}
__device__ __forceinline__ float2 ld_shared8(uint32_t saddr) {
  float2 v;
  asm volatile("ld.shared.v2.f32 {%0, %1}, [%2];" : "=f"(v.x), "=f"(v.y) : "r"(saddr) : "memory");
  return v;
}
// CLUSTER: what the other CTA of the pair wrote before it arrived is visible afterwards
struct Waiter {
  volatile uint32_t* abort_flag;
  template <bool CLUSTER = false>
  __device__ __forceinline__ bool on(uint64_t* bar, uint32_t parity) const {
    auto ready = [&]() { return CLUSTER ? tc::mbar_try_wait_cluster(bar, parity) : tc::mbar_try_wait(bar, parity); };
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

// VEC4: float32 matrices whose rows are X's rows and multiples of 16 bytes; else any type, order and alignment.
template <int MODE, bool VEC4>
__global__ void __launch_bounds__(Cfg<MODE>::THREADS, Cfg<MODE>::PER_SM) ns_on_chip(const NsJob J) {
  using C = Cfg<MODE>;
  constexpr bool PAIR = C::PAIR;
  constexpr int kWorkWarps = C::WORK, kMmaWarp = C::WORK, kSideWarp = C::WORK + 1, SUBS = C::SUBS;
  extern __shared__ __align__(1024) uint8_t smem_raw[];
  const uint32_t sbase = (tc::smem_u32(smem_raw) + 1023u) & ~1023u;
  const uint32_t sX = sbase, sA = sbase + C::X_BYTES;
  uint8_t* gen = smem_raw + (sbase - tc::smem_u32(smem_raw));
  Bars* B = reinterpret_cast<Bars*>(gen + C::X_BYTES + C::A_BYTES);
  uint32_t* tmem_slot = reinterpret_cast<uint32_t*>(B + 1);
  volatile uint32_t* abort_flag = tmem_slot + 1;
  double* sums = reinterpret_cast<double*>(gen + C::X_BYTES + C::A_BYTES + 512);   // [16] own warps, [2] the partner's total

  if (C::SLACK == 0 && sbase != tc::smem_u32(smem_raw)) {  // the base is not where it has to be: nothing fits
    if (threadIdx.x == 0) atomicMin(J.status, (int32_t)GNNCO_INTERNAL);
    return;
  }
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const uint32_t rank = PAIR ? tc::cluster_ctarank() : 0u;
  const int64_t group = blockIdx.x / C::CTAS, groups = gridDim.x / C::CTAS;
  const int kc = (J.k + 15) / 16 * 16, nc = (J.n + 15) / 16 * 16;   // contraction lengths
  const int a_items = (kc + 31) / 32, x_items = (nc + 31) / 32;     // 32-column items of A / P and of X
  const int quarters = PAIR ? 4 : (J.k + 31) / 32;                  // row quarters that hold anything
  const Waiter waiter{abort_flag};
  auto wait = [&](uint64_t* bar, uint32_t parity) { return waiter.on<false>(bar, parity); };
  auto wait_both = [&](uint64_t* bar, uint32_t parity) { return waiter.on<PAIR>(bar, parity); };

  if (threadIdx.x == 0) {
    auto panel_items = [](int items, int p) { const int left = items - 2 * p; return left <= 0 ? 1 : left >= 2 ? 2 : left; };
    for (int p = 0; p < 4; ++p) {
      tc::mbar_init(&B->x[p], quarters * panel_items(x_items, p) * C::CTAS);
      tc::mbar_init(&B->a[p], quarters * panel_items(a_items, p) * C::CTAS);
      tc::mbar_init(&B->p[p], quarters * panel_items(a_items, p) * C::CTAS);
    }
    tc::mbar_init(&B->m1, 1); tc::mbar_init(&B->m2, 1); tc::mbar_init(&B->m3, 1); tc::mbar_init(&B->lofree, 1);
    tc::mbar_init(&B->l, quarters * (a_items > SUBS ? a_items - SUBS : 1) * C::CTAS);
    // items of the off-diagonal half that this CTA writes: the upper columns in the even CTA, the lower ones in the odd
    tc::mbar_init(&B->own, 4 * (rank == 0 ? (x_items > 4 ? x_items - 4 : 1) : 4));
    tc::mbar_init(&B->g, 1);
    tc::mbar_init(&B->s, 1); tc::mbar_init(&B->s2, 1);
    tc::mbar_init(&B->norm, kWorkWarps); tc::mbar_init(&B->again, kWorkWarps); tc::mbar_init(&B->loaded, kWorkWarps);
    tc::mbar_init(&B->peer1, 1); tc::mbar_init(&B->peer2, 1);
    *abort_flag = 0;
    tc::fence_mbar_init();
  }
  if (warp == 0) {
    if constexpr (PAIR) tc::tmem_alloc_pair(tmem_slot, C::TMEM);
    else tc::tmem_alloc(tmem_slot, C::TMEM);
  }
  tc::tc_fence_before_sync();
  __syncthreads();
  if constexpr (PAIR) tc::cluster_sync_all();
  tc::tc_fence_after_sync();
  const uint32_t tmem = *tmem_slot;
  // the exchange scratch of this pair: [CTA][limb][2 panels]
  uint8_t* const scratch = PAIR ? static_cast<uint8_t*>(J.scratch) + group * (2 * 4 * (int64_t)kPanel) : nullptr;

  // The last step has begun: its weights and the next matrix are brought into L2 meanwhile, by one thread (each CTA of a pair:
  // its half of the bytes; earlier, the lines of all CTAs together would not survive in L2).
  auto prefetch = [&](int64_t s) {
    if (!J.prefetch) return;
    const int64_t bytes = (int64_t)J.r * J.c * 4, cut = bytes / 32 * 16, next = s + groups;
    const int64_t lo = PAIR && rank == 1 ? cut : 0, hi = PAIR && rank == 0 ? cut : bytes;
    auto fetch = [&](const void* array, int64_t set) {
      for (int64_t at = lo; array && at < hi; at += 16384)
        tc::prefetch_l2(static_cast<const char*>(array) + set * bytes + at, (uint32_t)(hi - at < 16384 ? hi - at : 16384));
    };
    fetch(J.W, s);
    if (next < J.sets && !(J.active && !J.active[next])) {
      fetch(J.G, next);
      fetch(J.m, next);
    }
  };

  if (warp == kMmaWarp) {
    // ------------------------------------------------------------------------------ MMA issue
    {
      // the whole warp takes every step together (see mma_f16); one lane issues
      const uint32_t leader = tc::elect_one();
      auto wait = [&](uint64_t* bar, uint32_t parity) { return __all_sync(0xffffffffu, waiter.on<false>(bar, parity)) != 0; };
      auto wait_both = [&](uint64_t* bar, uint32_t parity) { return __all_sync(0xffffffffu, waiter.on<PAIR>(bar, parity)) != 0; };
      const uint32_t i1 = tc::idesc_f16_f32(PAIR ? 256 : 128, PAIR ? 256 : kc, false);
      const uint32_t i3 = tc::idesc_f16_f32(PAIR ? 256 : 128, PAIR ? 256 : nc, true);
      auto commit = [&](uint64_t* bar) {
        if (leader) {
          if constexpr (PAIR) tc::mma_commit_pair(bar, 3);
          else tc::mma_commit(bar);
        }
        __syncwarp();
      };
      // Everything a product needs is a base plus constants, so that an MMA costs the issuing thread a few instructions:
      // 16 of k are 32 bytes of a k-major row, 2,048 bytes of n-major rows and 8 columns of tensor memory.
      const uint64_t xh = tc::smem_desc_sw128(sX, 16, 1024), xl = tc::smem_desc_sw128(sX + C::XP * kPanel, 16, 1024);
      const uint64_t ah = tc::smem_desc_sw128(sA, 16, 1024), al = tc::smem_desc_sw128(sA + C::A_HI * kPanel, 16, 1024);
      const uint64_t nh = tc::smem_desc_sw128(sX, kPanel, 1024), nl = tc::smem_desc_sw128(sX + C::XP * kPanel, kPanel, 1024);
      constexpr uint64_t kDescPanel = kPanel >> 4;
      auto n_off = [](int p) {                             // rows 64 p .. of X: in a pair rows 128 .. are in panels 2 and 3
        return (uint64_t)((PAIR ? (p >> 1) * 2 * kPanel + (p & 1) * 8192u : (uint32_t)p * 8192u) >> 4);
      };
      const int tk = kc / 16, tn = nc / 16;                // k-steps of 16
      // k-steps of panel p: f(step inside the panel)
      auto steps_of = [](int p, int t_end, auto f) {
#pragma unroll
        for (int q = 0; q < 4; ++q)
          if (4 * p + q < t_end) f(q);
      };
      const uint32_t tbase = __shfl_sync(0xffffffffu, tmem, 0);
      const uint32_t acc1 = tbase + C::ACC1, acc2 = tbase + C::ACC2, acc3 = tbase + C::ACC3;
      auto lefth = [&](int p, int q) { return (uint64_t)(acc1 + p * 64 + (q >> 1) * 32 + (q & 1) * 8); };
      auto leftl = [&](int p, int q) { return lefth(p, q) + 16; };
      uint32_t it = 0;
      for (int64_t s = group; s < J.sets; s += groups) {
        if (J.active && !J.active[s]) continue;
        bool ok = true;
        for (int step = 0; step < J.steps && ok; ++step, ++it) {
          const uint32_t ph = it & 1;
          if (rank == 0) {                                 // X X^T
            for (int p = 0; 4 * p < tn && ok; ++p) {
              ok = wait_both(&B->x[p], ph);
              tc::tc_fence_after_sync();
              if (ok) steps_of(p, tn, [&](int q) {
                const uint64_t o = p * kDescPanel + 2 * q;
                tc::mma_f16<PAIR, false>(leader, acc1, xh + o, xl + o, i1, p + q != 0);
                tc::mma_f16<PAIR, false>(leader, acc1, xl + o, xh + o, i1, true);
              });
            }
            if (!ok) break;
            for (int p = 0; 4 * p < tn; ++p)
              steps_of(p, tn, [&](int q) {
                const uint64_t o = p * kDescPanel + 2 * q;
                tc::mma_f16<PAIR, false>(leader, acc1, xh + o, xh + o, i1, true);
              });
            commit(&B->m1);
            if (!PAIR && leader && step == J.steps - 1) prefetch(s);
            __syncwarp();
          }
          if (rank == 0) {
            if constexpr (C::LATE) {                       // A A: what reads the first half of A's low limb comes first
              for (int p = 0; p < C::A_LO && ok; ++p) {
                ok = wait_both(&B->a[p], ph);
                tc::tc_fence_after_sync();
                if (ok) steps_of(p, tk, [&](int q) { tc::mma_f16<PAIR, true>(leader, acc2, lefth(p, q), al + p * kDescPanel + 2 * q, i1, p + q != 0); });
              }
              if (!ok) break;
              commit(&B->lofree);
            }
            for (int p = 0; 4 * p < tk && ok; ++p) {
              if (!C::LATE || p >= C::A_LO) {
                ok = wait_both(&B->a[p], ph);
                tc::tc_fence_after_sync();
              }
              if (ok) steps_of(p, tk, [&](int q) {
                const uint64_t o = p * kDescPanel + 2 * q;
                tc::mma_f16<PAIR, true>(leader, acc2, leftl(p, q), ah + o, i1, C::LATE || p + q != 0);
                if constexpr (!C::LATE) tc::mma_f16<PAIR, true>(leader, acc2, lefth(p, q), al + o, i1, true);
              });
            }
            if (C::LATE && 4 * C::A_LO < tk) {
              ok = ok && wait_both(&B->l, ph);
              tc::tc_fence_after_sync();
              for (int p = C::A_LO; 4 * p < tk && ok; ++p)
                steps_of(p, tk, [&](int q) { tc::mma_f16<PAIR, true>(leader, acc2, lefth(p, q), al + (p - C::A_LO) * kDescPanel + 2 * q, i1, true); });
            }
            if (!ok) break;
            for (int p = 0; 4 * p < tk; ++p)
              steps_of(p, tk, [&](int q) { tc::mma_f16<PAIR, true>(leader, acc2, lefth(p, q), ah + p * kDescPanel + 2 * q, i1, true); });
            commit(&B->m2);
            // P X.  Where the accumulator is the one A A is read from, all of P must be there.
            if constexpr (C::SHARED_ACC) {
              for (int p = 0; 4 * p < tk; ++p) ok = ok && wait_both(&B->p[p], ph);
              if (PAIR) ok = ok && wait(&B->s, ph) && wait_both(&B->s2, ph);
              tc::tc_fence_after_sync();
            }
            for (int p = 0; 4 * p < tk && ok; ++p) {
              if (!C::SHARED_ACC) {
                ok = wait(&B->p[p], ph);
                tc::tc_fence_after_sync();
              }
              if (ok) steps_of(p, tk, [&](int q) {
                const uint64_t o = n_off(p) + 128 * q;
                tc::mma_f16<PAIR, true>(leader, acc3, lefth(p, q), nl + o, i3, p + q != 0);
                tc::mma_f16<PAIR, true>(leader, acc3, leftl(p, q), nh + o, i3, true);
              });
            }
            if (!ok) break;
            for (int p = 0; 4 * p < tk; ++p)
              steps_of(p, tk, [&](int q) { tc::mma_f16<PAIR, true>(leader, acc3, lefth(p, q), nh + n_off(p) + 128 * q, i3, true); });
            commit(&B->m3);
          }
        }
        if (!ok) break;
      }
    }
    __syncwarp();
  } else if (PAIR && warp == kSideWarp) {
    // ------------------------------------------------------------------------------ exchange
    if (lane == 0) {
      uint32_t it = 0;
      bool ok = true;
      for (int64_t s = group; s < J.sets && ok; s += groups) {
        if (J.active && !J.active[s]) continue;
        for (int step = 0; step < J.steps && ok; ++step, ++it) {
          const uint32_t ph = it & 1;
          if (step == J.steps - 1) prefetch(s);
          const uint32_t mine = (rank == 0 ? 2 : 0) * kPanel;             // the two panels that change hands
          if (!(ok = wait(&B->own, ph))) break;
          for (int limb = 0; limb < 2; ++limb)
            tc::bulk_store(scratch + (rank * 2 + limb) * 2 * kPanel, sX + limb * C::XP * kPanel + mine, 2 * kPanel);
          tc::bulk_store_wait();
          tc::fence_proxy_async_all();
          tc::mbar_arrive_release_cluster(tc::map_to_cta(tc::smem_u32(&B->g), rank ^ 1u));
          // X X^T has read the rows: the block gives way to the partner's
          if (!(ok = wait(&B->m1, ph) && wait_both(&B->g, ph))) break;
          tc::fence_proxy_async_all();
          tc::mbar_arrive_expect_tx(&B->s, 4 * kPanel);
          for (int limb = 0; limb < 2; ++limb)
            tc::bulk_load(sX + limb * C::XP * kPanel + mine, scratch + ((rank ^ 1u) * 2 + limb) * 2 * kPanel, 2 * kPanel, &B->s);
          if (!(ok = wait(&B->s, ph))) break;
          if (rank == 1) tc::mbar_arrive_release_cluster(tc::map_to_cta(tc::smem_u32(&B->s2), 0));
        }
      }
    }
    __syncwarp();
  } else {
    // ------------------------------------------------------------------------------ load, convert, store
    const int quarter = warp & 3, sub = warp >> 2;
    const int row = quarter * 32 + lane;                   // of this CTA's 128
    const uint32_t lanes = (uint32_t)(quarter * 32) << 16;
    const bool works = quarter < quarters;
    // A warp without an item of X has none of A and P either, and nobody waits for it inside a step: it keeps away from the steps'
    // barriers (one that completed twice while it was on its way would look as if it had not completed).
    const bool busy = works && sub < x_items;
    const int off_panel = rank == 0 ? 2 : 0;               // the two panels that the partner takes
    auto arrive = [&](uint64_t* bar) {                     // on the even CTA's barrier, by one lane, after __syncwarp
      if constexpr (PAIR) tc::mbar_arrive_cluster(tc::map_to_cta(tc::smem_u32(bar), 0));
      else tc::mbar_arrive(bar);
    };
    // an item of X is written: tell the issuer, and the side warp where the partner needs it
    auto x_ready = [&](int item) {
      if (!works || item >= x_items || lane != 0) return;
      arrive(&B->x[item >> 1]);
      if (PAIR && ((item >> 1) & 2) == off_panel) tc::mbar_arrive(&B->own);
    };
    // chunk: 8 columns, counted over the row
    auto put_chunk = [&](int limb, int r, int chunk, const uint32_t* v) {
      tc::st_shared16(sX + (limb * C::XP + (chunk >> 3)) * kPanel + at_chunk(r, chunk & 7), v[0], v[1], v[2], v[3]);
    };
    // the loader's unit: 4 columns of a row, 8 bytes in each limb
    auto unit_at = [&](int limb, int r, int unit) {
      return sX + (limb * C::XP + (unit >> 4)) * kPanel + at_chunk(r, (unit >> 1) & 7) + (unit & 1) * 8;
    };
    const int upr = (nc + 31) / 32 * 8;                    // units per row that are kept (whole items)
    const int rows_kept = quarters * 32, total = rows_kept * upr;
    constexpr int kStride = 32 * kWorkWarps;
    // units are dealt along the matrix' own rows, so that lanes read neighbouring addresses
    const bool by_row = VEC4 || !J.transpose;
    const int per = by_row ? upr : rows_kept, jump_a = kStride / per, jump_b = kStride - jump_a * per;
    const int first_a = (int)threadIdx.x / per, first_b = (int)threadIdx.x - first_a * per;
    auto next_unit = [&](int& a, int& b) {                 // kStride units on
      a += jump_a;
      b += jump_b;
      if (b >= per) { b -= per; ++a; }
    };
    uint32_t it = 0, mat = 0, sum_it = 0, second_it = 0, again_it = 0;
    for (int64_t s = group; s < J.sets && !*abort_flag; s += groups) {
      if (J.active && !J.active[s]) continue;
      const int64_t base = s * (int64_t)J.r * J.c;
      const float* const Gs = static_cast<const float*>(J.G) + base;
      float* const Ms = J.m ? J.m + base : nullptr;
      float* const Ws = J.W ? J.W + base : nullptr;
      // the last matrix' values have left the room they were staged in
      __syncwarp();
      if (lane == 0) tc::mbar_arrive(&B->again);
      if (!wait(&B->again, again_it++ & 1)) break;
      // ---- momentum, u, |u|^2.  A unit (four columns of a row) of u waits as float32 in the two 8-byte places that its limbs
      // will take; four units (two where elements come one by one) are asked for at a time.
      double sum = 0.0;
      int ua = first_a, ub = first_b;
      constexpr int kUnits = VEC4 ? 4 : 2;
      for (int q = threadIdx.x; q < total; q += kUnits * kStride) {
        float g[kUnits][4], mv[kUnits][4];
        int at[kUnits];                                         // unit's offset in the matrix, -1: outside
        uint32_t place[kUnits];                                 // ... and its place in the high limb
#pragma unroll
        for (int y = 0; y < kUnits; ++y) {
          const int r = by_row ? ua : ub, unit = by_row ? ub : ua;
          next_unit(ua, ub);
          const int i = (int)rank * 128 + r, j = unit * 4;
          at[y] = q + y * kStride >= total || i >= J.k || j >= J.n ? -1 : by_row ? i * J.c + j : j * J.c + i;
          place[y] = unit_at(0, r, unit);
#pragma unroll
          for (int e = 0; e < 4; ++e) g[y][e] = mv[y][e] = 0.0f;
          if (at[y] < 0) continue;
          if constexpr (VEC4) {
            const float4 a = __ldcs(reinterpret_cast<const float4*>(Gs + at[y]));
            g[y][0] = a.x; g[y][1] = a.y; g[y][2] = a.z; g[y][3] = a.w;
            if (Ms) {
              const float4 b = __ldcs(reinterpret_cast<const float4*>(Ms + at[y]));
              mv[y][0] = b.x; mv[y][1] = b.y; mv[y][2] = b.z; mv[y][3] = b.w;
            }
          } else {
            const int hop = by_row ? 1 : J.c, have = J.n - j;
#pragma unroll
            for (int e = 0; e < 4; ++e)
              if (e < have) {
                g[y][e] = J.g_bf16 ? __bfloat162float(static_cast<const __nv_bfloat16*>(J.G)[base + at[y] + e * hop]) : __ldcs(Gs + at[y] + e * hop);
                if (Ms) mv[y][e] = __ldcs(Ms + at[y] + e * hop);
              }
          }
        }
#pragma unroll
        for (int y = 0; y < kUnits; ++y) {
          if (q + y * kStride >= total) continue;
          if (Ms && at[y] >= 0) {
#pragma unroll
            for (int e = 0; e < 4; ++e) {
              mv[y][e] = J.mu * mv[y][e] + g[y][e];
              g[y][e] = J.nesterov ? g[y][e] + J.mu * mv[y][e] : mv[y][e];
            }
            if constexpr (VEC4) {
              __stcs(reinterpret_cast<float4*>(Ms + at[y]), make_float4(mv[y][0], mv[y][1], mv[y][2], mv[y][3]));
            } else {
              const int hop = by_row ? 1 : J.c, have = J.n - (by_row ? at[y] % J.c : at[y] / J.c);
#pragma unroll
              for (int e = 0; e < 4; ++e)
                if (e < have) __stcs(Ms + at[y] + e * hop, mv[y][e]);
            }
          }
          // float32 squares of four values at a time, float64 across; the few matrices whose squares leave float32's range
          // are summed again below
          sum += (double)(g[y][0] * g[y][0] + g[y][1] * g[y][1] + g[y][2] * g[y][2] + g[y][3] * g[y][3]);
          st_shared8(place[y], __float_as_uint(g[y][0]), __float_as_uint(g[y][1]));
          st_shared8(place[y] + C::XP * kPanel, __float_as_uint(g[y][2]), __float_as_uint(g[y][3]));
        }
      }
      double norm2 = 0.0;
      // own warps' sums in warp order, then the partner's (a + b = b + a: both CTAs get the same bits).  Nothing in the partner
      // waits for this CTA's warps between the two rounds of a matrix, so each round has a barrier of its own: one that
      // completed twice while a warp was on its way to it would look as if it had not completed.
      auto total_of = [&](double part, uint64_t* peer_bar, uint32_t peer_parity) {
#pragma unroll
        for (int d = 16; d > 0; d >>= 1) part += __shfl_xor_sync(0xffffffffu, part, d);
        if (lane == 0) {
          sums[warp] = part;
          tc::mbar_arrive(&B->norm);
        }
        if (!wait(&B->norm, sum_it & 1)) return false;
        norm2 = 0.0;
#pragma unroll
        for (int w = 0; w < kWorkWarps; ++w) norm2 += sums[w];
        if constexpr (PAIR) {
          if (threadIdx.x == 0) {
            const uint32_t peer = tc::map_to_cta(tc::smem_u32(sums + 16 + (sum_it & 1)), rank ^ 1u);
            asm volatile("st.shared::cluster.f64 [%0], %1;" ::"r"(peer), "d"(norm2) : "memory");
            tc::mbar_arrive_release_cluster(tc::map_to_cta(tc::smem_u32(peer_bar), rank ^ 1u));
          }
          if (!wait_both(peer_bar, peer_parity)) return false;
          norm2 += sums[16 + (sum_it & 1)];
        }
        ++sum_it;
        return true;
      };
      if (!total_of(sum, &B->peer1, mat & 1)) break;
      if (!(norm2 > 1e-24 && norm2 < 1e37)) {              // the same decision everywhere
        // everybody has read the sums of the first round before they are written again
        __syncwarp();
        if (lane == 0) tc::mbar_arrive(&B->again);
        if (!wait(&B->again, again_it++ & 1)) break;
        sum = 0.0;
        int a2 = first_a, b2 = first_b;
        for (int q = threadIdx.x; q < total; q += kStride, next_unit(a2, b2)) {
          const uint32_t p = by_row ? unit_at(0, a2, b2) : unit_at(0, b2, a2);
          const float2 x = ld_shared8(p), y = ld_shared8(p + C::XP * kPanel);
          sum += (double)x.x * x.x + (double)x.y * x.y + ((double)y.x * y.x + (double)y.y * y.y);
        }
        if (!total_of(sum, &B->peer2, second_it++ & 1)) break;
      }
      const NsFactor by = ns_factor(norm2, J.eps, kXScale);
      if (by.lift != 1.0f) {                               // in place: every unit stays with its thread
        ua = first_a;
        ub = first_b;
        for (int q = threadIdx.x; q < total; q += kStride, next_unit(ua, ub)) {
          const uint32_t p = by_row ? unit_at(0, ua, ub) : unit_at(0, ub, ua);
          const float2 x = ld_shared8(p), y = ld_shared8(p + C::XP * kPanel);
          st_shared8(p, __float_as_uint(x.x * by.lift), __float_as_uint(x.y * by.lift));
          st_shared8(p + C::XP * kPanel, __float_as_uint(y.x * by.lift), __float_as_uint(y.y * by.lift));
        }
      }
      const float f = by.f;
      ua = first_a;
      ub = first_b;
#pragma unroll 4
      for (int q = threadIdx.x; q < total; q += kStride, next_unit(ua, ub)) {
        const uint32_t p = by_row ? unit_at(0, ua, ub) : unit_at(0, ub, ua);
        const float2 x = ld_shared8(p), y = ld_shared8(p + C::XP * kPanel);
        uint32_t hi[2], lo[2];
        split2(x.x * f, x.y * f, hi[0], lo[0]);
        split2(y.x * f, y.y * f, hi[1], lo[1]);
        st_shared8(p, hi[0], hi[1]);
        st_shared8(p + C::XP * kPanel, lo[0], lo[1]);
      }
      tc::fence_proxy_async_smem();
      __syncwarp();
      if (lane == 0) tc::mbar_arrive(&B->loaded);
      if (!wait(&B->loaded, mat & 1)) break;
      for (int item = sub; item < 2 * C::XP; item += SUBS) x_ready(item);

      bool ok = true;
      for (int step = 0; step < J.steps && busy; ++step, ++it) {
        const uint32_t ph = it & 1;
        // ---- A's limbs over its accumulator, and into shared memory
        if (!(ok = wait(&B->m1, ph))) break;
        tc::tc_fence_after_sync();
        uint32_t hi[16], lo[16];
        for (int item = sub; item < a_items; item += SUBS) {
          if (!works) break;
          uint32_t v[32];
          tc::tmem_ld_32x32(tmem + C::ACC1 + lanes + item * 32, v);
          tc::tmem_ld_wait();
          const uint64_t f1 = pair_of(kAScale / (kXScale * kXScale), kAScale / (kXScale * kXScale));
#pragma unroll
          for (int e = 0; e < 16; ++e) split2_scaled(v[2 * e], v[2 * e + 1], f1, hi[e], lo[e]);
          tc::tmem_st_32x16(tmem + C::ACC1 + lanes + item * 32, hi);
          tc::tmem_st_32x16(tmem + C::ACC1 + lanes + item * 32 + 16, lo);
          const int panel = item >> 1, c0 = (item & 1) * 4;
#pragma unroll
          for (int e = 0; e < 4; ++e)
            tc::st_shared16(sA + panel * kPanel + at_chunk(row, c0 + e), hi[4 * e], hi[4 * e + 1], hi[4 * e + 2], hi[4 * e + 3]);
          if (!C::LATE || panel < C::A_LO) {
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
        if (C::LATE) {
          // the low limb's second half, still in registers, follows into the room of the first
          if (!(ok = wait(&B->lofree, ph))) break;
          const int item = sub + SUBS;
          if (works && item < a_items) {
#pragma unroll
            for (int e = 0; e < 4; ++e)
              tc::st_shared16(sA + (C::A_HI + (item >> 1) - C::A_LO) * kPanel + at_chunk(row, (item & 1) * 4 + e), lo[4 * e], lo[4 * e + 1],
                              lo[4 * e + 2], lo[4 * e + 3]);
            tc::fence_proxy_async_smem();
            __syncwarp();
            if (lane == 0) arrive(&B->l);
          }
        }
        // ---- P = a I + b A + c A A over A's limbs
        if (!(ok = wait(&B->m2, ph))) break;
        tc::tc_fence_after_sync();
        const float fi = J.a * J.p_scale, fa1 = J.b * J.p_scale / kAScale, faa1 = J.cc * J.p_scale / (kAScale * kAScale);
        const uint64_t fa = pair_of(fa1, fa1), faa = pair_of(faa1, faa1);
        for (int item = sub; item < a_items; item += SUBS) {
          if (!works) break;
          uint32_t v[32];
          tc::tmem_ld_32x32(tmem + C::ACC2 + lanes + item * 32, v);
          tc::tmem_ld_32x16(tmem + C::ACC1 + lanes + item * 32, hi);
          tc::tmem_ld_32x16(tmem + C::ACC1 + lanes + item * 32 + 16, lo);
          tc::tmem_ld_wait();
#pragma unroll
          for (int e = 0; e < 16; ++e) {
            const float2 A2 = join2(hi[e], lo[e]);
            float p0, p1;
            unpair(fma2(fa, pair_of(A2.x, A2.y), mul2(faa, pair_of(__uint_as_float(v[2 * e]), __uint_as_float(v[2 * e + 1])))), p0, p1);
            v[2 * e] = __float_as_uint(p0);
            v[2 * e + 1] = __float_as_uint(p1);
          }
          if (item == (int)rank * 4 + quarter) {           // the item that holds the diagonal of these rows
#pragma unroll
            for (int e = 0; e < 32; ++e)
              if (e == lane) v[e] = __float_as_uint(__uint_as_float(v[e]) + fi);
          }
#pragma unroll
          for (int e = 0; e < 16; ++e) split2(__uint_as_float(v[2 * e]), __uint_as_float(v[2 * e + 1]), hi[e], lo[e]);
          tc::tmem_st_32x16(tmem + C::ACC1 + lanes + item * 32, hi);
          tc::tmem_st_32x16(tmem + C::ACC1 + lanes + item * 32 + 16, lo);
          tc::tmem_st_wait();
          tc::tc_fence_before_sync();
          __syncwarp();
          if (lane == 0) arrive(&B->p[item >> 1]);
        }
        // ---- X' over X
        if (step < J.steps - 1) {
          if (!(ok = wait(&B->m3, ph))) break;
          tc::tc_fence_after_sync();
          const uint64_t f3 = pair_of(1.0f / J.p_scale, 1.0f / J.p_scale);
          for (int item = sub; item < x_items; item += SUBS) {
            if (!works) break;
            uint32_t v[32];
            tc::tmem_ld_32x32(tmem + C::ACC3 + lanes + item * 32, v);
            tc::tmem_ld_wait();
#pragma unroll
            for (int e = 0; e < 16; ++e) split2_scaled(v[2 * e], v[2 * e + 1], f3, hi[e], lo[e]);
#pragma unroll
            for (int e = 0; e < 4; ++e) {
              put_chunk(0, row, item * 4 + e, hi + 4 * e);
              put_chunk(1, row, item * 4 + e, lo + 4 * e);
            }
            tc::fence_proxy_async_smem();
            tc::tc_fence_before_sync();
            __syncwarp();
            x_ready(item);
          }
          continue;
        }
        // ---- the last step: into the weights (or the result).  Values of W are asked for before they are needed; rows pass
        // through this warp's 4 KB of X's room, so that lanes work on neighbouring addresses.
        const float fo = 1.0f / (J.p_scale * kXScale), keep = J.keep, step_w = J.step;
        const uint32_t stage = sX + warp * 4096;
        bool waited = false;
        auto first_wait = [&]() {                          // of the products that the last step ends with
          if (!waited) ok = wait(&B->m3, ph);
          if (ok && !waited) tc::tc_fence_after_sync();
          waited = true;
          return ok;
        };
        for (int item = sub; item < 2 * C::XP && ok; item += SUBS) {
          const bool in = works && item < x_items;
          if constexpr (VEC4) {
            // 4 columns of every fourth row
            const int i0 = (int)rank * 128 + quarter * 32 + (lane >> 3), j0 = item * 32 + (lane & 7) * 4, hop = 4 * J.c;
            const int have = in && i0 < J.k && j0 < J.n ? (J.k - i0 + 3) / 4 : 0, at = i0 * J.c + j0;
            float4 w[8];
            if (Ws) {
#pragma unroll
              for (int e = 0; e < 8; ++e)
                w[e] = e < have ? __ldcs(reinterpret_cast<const float4*>(Ws + at + e * hop)) : make_float4(0.0f, 0.0f, 0.0f, 0.0f);
            }
            if (!first_wait()) break;
            if (!in) continue;
            {
              uint32_t v[32];
              tc::tmem_ld_32x32(tmem + C::ACC3 + lanes + item * 32, v);
              tc::tmem_ld_wait();
#pragma unroll
              for (int e = 0; e < 8; ++e) tc::st_shared16(stage + at_chunk(lane, e), v[4 * e], v[4 * e + 1], v[4 * e + 2], v[4 * e + 3]);
            }
            __syncwarp();
#pragma unroll
            for (int e = 0; e < 8; ++e) {
              const uint4 a = tc::ld_shared16(stage + at_chunk(4 * e + (lane >> 3), lane & 7));
              if (e >= have) continue;
              float x[4] = {__uint_as_float(a.x) * fo, __uint_as_float(a.y) * fo, __uint_as_float(a.z) * fo, __uint_as_float(a.w) * fo};
              if (Ws) {
                x[0] = w[e].x * keep - step_w * x[0];
                x[1] = w[e].y * keep - step_w * x[1];
                x[2] = w[e].z * keep - step_w * x[2];
                x[3] = w[e].w * keep - step_w * x[3];
              }
              if (Ws || !J.o_bf16) {
                __stcs(reinterpret_cast<float4*>((Ws ? Ws : static_cast<float*>(J.O) + base) + at + e * hop), make_float4(x[0], x[1], x[2], x[3]));
              } else {
                __stcs(reinterpret_cast<uint2*>(static_cast<__nv_bfloat16*>(J.O) + base + at + e * hop),
                       make_uint2(vio::pack_bf16(x[0], x[1]), vio::pack_bf16(x[2], x[3])));
              }
            }
            __syncwarp();
          } else {
            // rows of W: the item's 32 rows at one column per lane; columns of W (transposed): its 32 columns at one row of X per
            // lane; 16 at a time
            const int i0 = (int)rank * 128 + quarter * 32 + (J.transpose ? lane : 0), j0 = item * 32 + (J.transpose ? 0 : lane);
            int have = 0;
            if (in && i0 < J.k && j0 < J.n) have = J.transpose ? J.n - j0 : J.k - i0;
            const int at0 = J.transpose ? j0 * J.c + i0 : i0 * J.c + j0;
            if (!J.transpose) {
              if (!first_wait()) break;
              if (in) {
#pragma unroll
                for (int hf = 0; hf < 2; ++hf) {
                  uint32_t v[16];
                  tc::tmem_ld_32x16(tmem + C::ACC3 + lanes + item * 32 + hf * 16, v);
                  tc::tmem_ld_wait();
#pragma unroll
                  for (int e = 0; e < 4; ++e) tc::st_shared16(stage + at_chunk(lane, hf * 4 + e), v[4 * e], v[4 * e + 1], v[4 * e + 2], v[4 * e + 3]);
                }
                __syncwarp();
              }
            }
#pragma unroll 1
            for (int hf = 0; hf < 2; ++hf) {
              const int at = at0 + hf * 16 * J.c, left = have - hf * 16;
              float w[16];
              uint32_t v[16];
#pragma unroll
              for (int e = 0; e < 16; ++e) w[e] = Ws && e < left ? __ldcs(Ws + at + e * J.c) : 0.0f;
              if (!first_wait()) break;
              if (!in) break;
              if (J.transpose) {
                tc::tmem_ld_32x16(tmem + C::ACC3 + lanes + item * 32 + hf * 16, v);
                tc::tmem_ld_wait();
              } else {
#pragma unroll
                for (int e = 0; e < 16; ++e)
                  asm volatile("ld.shared.b32 %0, [%1];" : "=r"(v[e]) : "r"(stage + at_chunk(hf * 16 + e, lane >> 2) + (lane & 3) * 4) : "memory");
              }
#pragma unroll
              for (int e = 0; e < 16; ++e) {
                if (e >= left) continue;
                const float x = __uint_as_float(v[e]) * fo;
                if (Ws) __stcs(Ws + at + e * J.c, w[e] * keep - step_w * x);
                else if (J.o_bf16) static_cast<__nv_bfloat16*>(J.O)[base + at + e * J.c] = __float2bfloat16_rn(x);
                else __stcs(static_cast<float*>(J.O) + base + at + e * J.c, x);
              }
            }
            __syncwarp();
          }
        }
        if (!ok) break;
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
    if (warp == 0) tc::tmem_dealloc_pair(tmem, C::TMEM);
  } else {
    if (warp == 0) tc::tmem_dealloc(tmem, C::TMEM);
  }
}

template <int MODE>
void launch_shape(cudaLaunchConfig_t& cfg, cudaLaunchAttribute* attr, int ctas, cudaStream_t st) {
  cfg.gridDim = dim3(ctas);
  cfg.blockDim = dim3(Cfg<MODE>::THREADS);
  cfg.dynamicSmemBytes = Cfg<MODE>::SMEM;
  cfg.stream = st;
  attr[0].id = cudaLaunchAttributeClusterDimension;
  attr[0].val.clusterDim.x = Cfg<MODE>::CTAS;
  attr[0].val.clusterDim.y = attr[0].val.clusterDim.z = 1;
  cfg.attrs = attr;
  cfg.numAttrs = 1;
}

// CTA pairs that can be resident at once (asked once per process; 0: none)
int resident_pairs() {
  static const int pairs = [] {
    if (cudaFuncSetAttribute((ns_on_chip<kPair, true>), cudaFuncAttributeMaxDynamicSharedMemorySize, (int)Cfg<kPair>::SMEM) != cudaSuccess) {
      cudaGetLastError();
      return 0;
    }
    cudaLaunchConfig_t cfg{};
    cudaLaunchAttribute attr[1];
    launch_shape<kPair>(cfg, attr, 2 * 148, nullptr);
    int n = 0;
    if (cudaOccupancyMaxActiveClusters(&n, (ns_on_chip<kPair, true>), &cfg) != cudaSuccess) {
      cudaGetLastError();
      n = 0;
    }
    return n;
  }();
  return pairs;
}

template <int MODE, bool VEC4>
int32_t launch(gnnco_handle* h, const NsJob& job, int64_t groups, cudaStream_t st) {
  static std::atomic<int> allowed{0};
  const int32_t rc = allow_shared_memory(ns_on_chip<MODE, VEC4>, Cfg<MODE>::SMEM, h->device, allowed);
  if (rc != GNNCO_OK) return rc;
  cudaLaunchConfig_t cfg{};
  cudaLaunchAttribute attr[1];
  if (groups > job.sets) groups = job.sets;
  launch_shape<MODE>(cfg, attr, (int)groups * Cfg<MODE>::CTAS, st);
  GNNCO_CUDA_TRY(cudaLaunchKernelEx(&cfg, (ns_on_chip<MODE, VEC4>), job));
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
  auto run = [&](auto mode, int64_t groups) {
    constexpr int MODE = decltype(mode)::value;
    return job.vec4 ? launch<MODE, true>(h, job, groups, st) : launch<MODE, false>(h, job, groups, st);
  };
  if (job.n <= 128) return run(std::integral_constant<int, kDual>(), 2 * (int64_t)h->sm_count);
  if (job.k <= 128) return run(std::integral_constant<int, kWide>(), h->sm_count);
  return run(std::integral_constant<int, kPair>(), resident_pairs());
}
