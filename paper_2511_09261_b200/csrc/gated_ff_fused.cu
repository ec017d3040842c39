// The gated feed-forward block's forward pass as ONE kernel, for bfloat16 operands and widths F, F_out <= 256: h never leaves the SM.
//
//   a cluster of two CTAs takes 256 rows of x, which stay in shared memory, and walks H in chunks of 128 columns:
//     G(c)   [g | u] = x [Wg | Wu]       256 x 256 in tensor memory
//     result warps   h = act(g) .* u     -> bfloat16, into shared memory, in the layout of an MMA operand
//     D(c)   y += h Wd                   256 x F_out, in tensor memory until the last chunk
//
// The products are issued G(0) G(1) D(0) G(2) D(1) .., across tiles too.  While D(c - 1) is multiplied the result warps take g and u of
// chunk c into registers, so that G(c + 1) finds its accumulator free, and they have that long to finish h (24 instructions of 128
// cycles a chunk at F = F_out = 256).  A tile's y is taken out after the first chunk of the next tile, for the same reason.  With dropout behind the
// block six more warps draw the words of y's elements meanwhile and leave one bit per element in shared memory: drawn by the
// result warps they took as long as everything else (2,230 us for 2.5 M x 256 x 512, against 1,950).
// (Chunks of 64 columns with two accumulators of g and u halved the work per instruction and reread x twice as often: 2,070 us for
// 2.5 M x 256 x 512 without dropout against 1,590.)
// The weights come from L2 again for every tile: 96 KB per chunk and CTA, 32 bytes a cycle (an SM gets some 45).  Against the two
// launches of gated_ff_tiles.cuh this saves writing and reading h, 4 H bytes per row of 4 F read and written.
// What bounds it: the products without dropout (400,000 x 256 x 512: 272 us, tensor pipe 63 % active, the special functions of SiLU 47 %),
// products and the words' wide multiplications with it (331 us, tensor pipe 50 %).  DRAM carries 1.9 TB/s.
//
// Shared memory per CTA: x 64 KB, h 32 KB, blocks of Wg (even CTA) or Wu (odd) 4 x 16 KB, of Wd 2 x 16 KB, staging 16 KB, bits of the
// mask 2 x 4 KB.
// Roles of the warps: 0 products, 1 copies, 4-11 results; with dropout 2, 3 and 12-15 draw.  (Eight result warps with 168 registers
// each hold nearly all of their g and u, so the accumulator is free soon; sixteen with 96 had to compute the first half before they
// could take the second, and the products waited: 1,666 us against 1,590.  With dropout the launch has 128 registers a thread.)
#include "gated_ff_tiles.cuh"

namespace ff {
namespace {

constexpr int kChunk = 128;                                // columns of h
constexpr int kXBlocks = 4, kGSlots = 4, kDSlots = 2;      // blocks of 64 of a contraction
constexpr uint32_t kBlockBytes = 16384;
constexpr uint32_t kX = 0, kH = kX + kXBlocks * kBlockBytes, kG = kH + 2 * kBlockBytes, kD = kG + kGSlots * kBlockBytes,
                   kStaging = kD + kDSlots * kBlockBytes;
constexpr int kResults = 8, kDrawers = 6;
constexpr uint32_t kMaskBytes = 8 * 128 * 4;               // a bit for each of 128 x 256 elements: [column group][row]
constexpr uint32_t kMask = kStaging + kResults * kStageBytes, kBars = kMask + 2 * kMaskBytes;
constexpr uint32_t kFusedSmem = 1024 + kBars + 512;
static_assert(kFusedSmem <= 232448, "fits one SM");
constexpr uint32_t kYColumn = 0, kGuColumn = 256;          // tensor memory: y; g, then u

// barriers; the even CTA's are used but for those that both CTAs wait on (every commit arrives in both)
struct Bars {
  uint64_t x_full[kXBlocks], x_empty[kXBlocks];
  uint64_t g_full[kGSlots], g_empty[kGSlots];
  uint64_t d_full[kDSlots], d_empty[kDSlots];
  uint64_t gu_full, gu_empty, h_full, h_empty, y_full, y_empty;
  uint64_t mask_full[2], mask_empty[2];                    // every CTA's own
  uint32_t tmem, abort_flag;
};

constexpr int fused_threads(bool masked) { return 32 * (kFirstEpi + kResults + (masked ? 4 : 0)); }

template <bool MASKED>
__global__ void __launch_bounds__(fused_threads(MASKED), 1) fused_forward(const __grid_constant__ Maps maps, const __grid_constant__ Args A) {
  extern __shared__ uint8_t smem_raw[];
  const uint32_t sbase = (tc::smem_u32(smem_raw) + 1023u) & ~1023u;
  uint8_t* gen = smem_raw + (sbase - tc::smem_u32(smem_raw));
  Bars& B = *reinterpret_cast<Bars*>(gen + kBars);
  volatile uint32_t* abort_flag = &B.abort_flag;
  asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const uint32_t rank = tc::cluster_ctarank();
  const int first = blockIdx.x / 2, step = gridDim.x / 2;
  const int x_blocks = (A.K[0] + 63) >> 6;                 // of F
  const int chunks = (A.K[1] + kChunk - 1) / kChunk;       // of H
  const int y_cols = A.cols > 128 ? 256 : 128;

  if (threadIdx.x == 0) {
    for (int i = 0; i < kXBlocks; ++i) {
      tc::mbar_init(B.x_full + i, 2);
      tc::mbar_init(B.x_empty + i, 1);
    }
    for (int i = 0; i < kGSlots; ++i) {
      tc::mbar_init(B.g_full + i, 2);
      tc::mbar_init(B.g_empty + i, 1);
    }
    for (int i = 0; i < kDSlots; ++i) {
      tc::mbar_init(B.d_full + i, 2);
      tc::mbar_init(B.d_empty + i, 1);
    }
    tc::mbar_init(&B.gu_full, 1);
    tc::mbar_init(&B.gu_empty, 2 * kResults);
    tc::mbar_init(&B.h_full, kResults + (rank == 0 ? 1 : 0));        // the odd CTA's is passed on as one arrival
    tc::mbar_init(&B.h_empty, 1);
    tc::mbar_init(&B.y_full, 1);
    tc::mbar_init(&B.y_empty, 2 * kResults);
    for (int i = 0; i < 2; ++i) {
      tc::mbar_init(B.mask_full + i, kDrawers);
      tc::mbar_init(B.mask_empty + i, kResults);
    }
    *abort_flag = 0;
    tc::fence_mbar_init();
  }
  if (warp == 0) tc::tmem_alloc_pair(&B.tmem, 512);
  tc::tc_fence_before_sync();
  __syncthreads();
  tc::cluster_sync_all();
  tc::tc_fence_after_sync();
  const uint32_t tmem = B.tmem;

  if (warp == kCopyWarp) {
    // -------------------------------------------------------------------------------- operands
    const uint32_t leader = tc::elect_one();
    const int rank_u = __shfl_sync(0xffffffffu, (int)rank, 0);
    auto even = [&](uint64_t* bar) { return tc::map_to_cta(tc::smem_u32(bar), 0); };
    auto wait = [&](uint64_t* bar, uint32_t parity) { return __all_sync(0xffffffffu, wait_bar(bar, parity, abort_flag)) != 0; };
    Walk<kDown, true, true, true> walk(A, first, step);
    asm volatile("griddepcontrol.wait;" ::: "memory");     // (as in gated_ff_tiles.cuh: everything else hangs on the copies)
    int slot = 0, d = 0;
    uint32_t g_phase = 1, d_phase = 1, x_phase = 1;        // the first round waits for nothing
    bool ok = true;
    int d_chunk = -1, d_set = 0;
    auto load_d = [&] {
      for (int kb = 0; kb < 2; ++kb) {
        if (!wait(B.d_empty + d, d_phase)) return false;
        expect_bytes<true>(leader, even(B.d_full + d), y_cols * 64);
        for (int i = 0; i < y_cols / 128; ++i)
          load_box_of_set<true>(leader, sbase + kD + d * kBlockBytes + i * 8192, &maps.b[2], rank_u * (y_cols / 2) + 64 * i,
                                d_chunk * kChunk + kb * 64, d_set, even(B.d_full + d));
        d ^= 1;
        if (d == 0) d_phase ^= 1;
      }
      return true;
    };
    while (walk.any() && ok) {
      const Tile T = walk.take();
      for (int c = 0; c < chunks && ok; ++c) {
        for (int kb = 0; kb < x_blocks && ok; ++kb) {
          if (c == 0) {
            if (!(ok = wait(B.x_empty + kb, x_phase))) break;
            expect_bytes<true>(leader, even(B.x_full + kb), 16384);
            load_box<true>(leader, sbase + kX + kb * 16384, &maps.a[0], kb * 64, T.row0 + rank_u * 128, 0, even(B.x_full + kb));
          }
          if (!(ok = wait(B.g_empty + slot, g_phase))) break;
          expect_bytes<true>(leader, even(B.g_full + slot), kBlockBytes);
          for (int i = 0; i < 2; ++i)
            load_box_of_set<true>(leader, sbase + kG + slot * kBlockBytes + i * 8192, &maps.b[rank_u], c * kChunk + 64 * i, kb * 64, T.set,
                                  even(B.g_full + slot));
          if (++slot == kGSlots) {
            slot = 0;
            g_phase ^= 1;
          }
        }
        // Wd of the chunk before
        if (ok && d_chunk >= 0) ok = load_d();
        d_chunk = c;
        d_set = T.set;
      }
      x_phase ^= 1;
    }
    if (ok && d_chunk >= 0) load_d();
    __syncwarp();
  } else if (warp == kMmaWarp) {
    // -------------------------------------------------------------------------------- products
    const int tiles_here = first < A.tiles ? (A.tiles - first + step - 1) / step : 0;
    const int32_t total = tiles_here * chunks;
    if (rank == 1 && tc::elect_one()) {
      // This CTA's h is ready: passed on to the CTA that multiplies, with a release at the scope of the cluster.  (That waits for
      // everything its thread has in flight: nothing here, but 1,650 cycles a chunk in the result warps.)
      for (int32_t i = 0; i < total; ++i) {
        if (!wait_bar(&B.h_full, (uint32_t)i & 1, abort_flag)) break;
        tc::mbar_arrive_release_cluster(tc::map_to_cta(tc::smem_u32(&B.h_full), 0));
      }
    }
    if (rank == 0 && tc::elect_one()) {
      const uint32_t g_idesc = tc::idesc_bf16_f32(256, 256, false, true), d_idesc = tc::idesc_bf16_f32(256, y_cols, false, true);
      int slot = 0, d = 0, gc = 0, dc = 0;                 // gc, dc: chunk of the tile that G and D are at
      uint32_t g_phase = 0, d_phase = 0, x_phase = 0, y_phase = 1;
      bool ok = true;
      for (int32_t i = 0; i <= total && ok; ++i) {
        if (i < total) {
          if (!(ok = wait_bar(&B.gu_empty, (uint32_t)(i & 1) ^ 1, abort_flag))) break;
          tc::tc_fence_after_sync();
          for (int kb = 0; kb < x_blocks; ++kb) {
            if (gc == 0 && !(ok = wait_bar(B.x_full + kb, x_phase, abort_flag))) break;
            if (!(ok = wait_bar(B.g_full + slot, g_phase, abort_flag))) break;
            tc::tc_fence_after_sync();
            const uint64_t a0 = tc::smem_desc_sw128(sbase + kX + kb * kBlockBytes, 16, 1024);
            const uint64_t b0 = tc::smem_desc_sw128(sbase + kG + slot * kBlockBytes, 8192, 1024);
            const int steps = min(4, (A.K[0] - kb * 64 + 15) >> 4);
#pragma unroll
            for (int k = 0; k < 4; ++k)
              if (k < steps) multiply<true>(tmem + kGuColumn, a0 + 2 * k, b0 + 128 * k, g_idesc, kb + k != 0);
            commit<true>(B.g_empty + slot);
            if (gc == chunks - 1) commit<true>(B.x_empty + kb);
            if (++slot == kGSlots) {
              slot = 0;
              g_phase ^= 1;
            }
          }
          if (!ok) break;
          commit<true>(&B.gu_full);
          if (++gc == chunks) {
            gc = 0;
            x_phase ^= 1;
          }
        }
        if (i > 0) {
          if (!(ok = wait_bar<true>(&B.h_full, (uint32_t)(i - 1) & 1, abort_flag))) break;
          if (dc == 0) {
            if (!(ok = wait_bar(&B.y_empty, y_phase, abort_flag))) break;
            y_phase ^= 1;
          }
          for (int kb = 0; kb < 2; ++kb) {
            if (!(ok = wait_bar(B.d_full + d, d_phase, abort_flag))) break;
            tc::tc_fence_after_sync();
            const uint64_t a0 = tc::smem_desc_sw128(sbase + kH + kb * kBlockBytes, 16, 1024);
            const uint64_t b0 = tc::smem_desc_sw128(sbase + kD + d * kBlockBytes, 8192, 1024);
            const int steps = min(4, (A.K[1] - dc * kChunk - kb * 64 + 15) >> 4);    // none where H ends before
#pragma unroll
            for (int k = 0; k < 4; ++k)
              if (k < steps) multiply<true>(tmem + kYColumn, a0 + 2 * k, b0 + 128 * k, d_idesc, dc + kb + k != 0);
            commit<true>(B.d_empty + d);
            d ^= 1;
            if (d == 0) d_phase ^= 1;
          }
          if (!ok) break;
          commit<true>(&B.h_empty);
          if (++dc == chunks) {
            dc = 0;
            commit<true>(&B.y_full);
          }
        }
      }
    }
  } else if (warp >= kFirstEpi && warp < kFirstEpi + kResults) {
    // --------------------------------------------------------------------------------- results
    const int e = warp - kFirstEpi, quarter = warp & 3, half = e >> 2;
    const uint32_t lanes = (uint32_t)(quarter * 32) << 16;
    const int row_in_cta = quarter * 32 + lane, warp_row = (int)rank * 128 + quarter * 32;
    const uint32_t gu_free = tc::map_to_cta(tc::smem_u32(&B.gu_empty), 0), y_free = tc::map_to_cta(tc::smem_u32(&B.y_empty), 0);
    float* const stage = reinterpret_cast<float*>(gen + kStaging + e * kStageBytes);
    const uint32_t stage_at = sbase + kStaging + e * kStageBytes;
    const uint32_t h_at = sbase + kH + half * kBlockBytes + row_in_cta * 128;
    uint32_t y_phase = 0, phase = 0;                       // phase: of the chunk
    bool ok = true;
    // the tile whose y is still to be taken out: its first row of this warp, how many the tile has from there on, its number here
    int32_t y_row0 = 0, y_rows = 0;
    uint32_t y_tile = 0;
    auto take_y = [&] {
      if (!wait_bar(&B.y_full, y_phase, abort_flag)) return false;
      y_phase ^= 1;
      tc::tc_fence_after_sync();
      if (MASKED && !wait_bar(B.mask_full + (y_tile & 1), (y_tile >> 1) & 1, abort_flag)) return false;
#pragma unroll
      for (int g = 0; g < 4; ++g) {
        const int c0 = (half + 2 * g) * 32;
        const bool in = c0 < A.cols;
        float f[32];
        if (in) {
          uint32_t r[32];
          tmem_load(tmem + kYColumn + lanes + c0, r);
          tc::tmem_ld_wait();
#pragma unroll
          for (int k = 0; k < 32; ++k) f[k] = __uint_as_float(r[k]);
        }
        if (g == 3) {
          tc::tc_fence_before_sync();
          __syncwarp();
          if (lane == 0) tc::mbar_arrive_cluster(y_free);
        }
        if (!in) continue;
        if (MASKED) {
          const uint32_t keep = reinterpret_cast<const uint32_t*>(gen + kMask + (y_tile & 1) * kMaskBytes)[(half + 2 * g) * 128 + row_in_cta];
#pragma unroll
          for (int k = 0; k < 32; ++k) f[k] = (keep >> k) & 1u ? f[k] * A.mask.scale : 0.0f;
        }
        if (A.y_vectors && y_rows >= 32) stage_limbs<1>(&maps.out[0], stage_at, lane, c0, y_row0, f);
        else store_rows<false>(stage, lane, y_rows, y_row0, c0, A.cols, A.y, A.y_ld, f);
      }
      if (MASKED) {
        __syncwarp();
        if (lane == 0) tc::mbar_arrive(B.mask_empty + (y_tile & 1));
      }
      ++y_tile;
      return true;
    };
    // the next tile's table entries arrive while this one is worked on
    int32_t next_row0 = 0, next_rows = 0;
    auto fetch = [&](int t) {
      if (t >= A.tiles) return;
      next_row0 = A.tile_row0 ? A.tile_row0[t] : t * 256;
      next_rows = A.tile_row0 ? A.tile_rows[t] : (int32_t)min((int64_t)256, A.rows - (int64_t)t * 256);
    };
    fetch(first);
    for (int t = first; t < A.tiles && ok; t += step) {
      for (int c = 0; c < chunks && ok; ++c, phase ^= 1) {
        if (!(ok = wait_bar(&B.gu_full, phase, abort_flag))) break;
        tc::tc_fence_after_sync();
        // g and u into registers, 16 columns at a time, and the accumulator back as soon as the last of four are there: the next products
        // wait for it.  (The last are asked for when the first have been used: all at once do not fit.)
        constexpr int kAhead = MASKED ? 2 : 3;
        uint32_t r[4][2][16], w[32];
        const uint32_t at = tmem + kGuColumn + lanes + half * 64;
        auto load = [&](int b) {
          tmem_load(at + 16 * b, r[b][0]);
          tmem_load(at + 128 + 16 * b, r[b][1]);
        };
        auto convert = [&](int b) {
          float f[2][16];
#pragma unroll
          for (int k = 0; k < 16; ++k) {
            f[0][k] = __uint_as_float(r[b][0][k]);
            f[1][k] = __uint_as_float(r[b][1][k]);
          }
          if (A.act == GNNCO_SILU) gate<false, GNNCO_SILU>(f, 1.0f);
          else if (A.act == GNNCO_GELU) gate<false, GNNCO_GELU>(f, 1.0f);
          else gate<false, GNNCO_RELU>(f, 1.0f);
#pragma unroll
          for (int k = 0; k < 8; ++k) w[8 * b + k] = vio::pack_bf16(f[0][2 * k], f[0][2 * k + 1]);
        };
#pragma unroll
        for (int b = 0; b < kAhead; ++b) load(b);
        tc::tmem_ld_wait();
#pragma unroll
        for (int b = kAhead; b < 4; ++b) {
          convert(b - kAhead);
          load(b);
        }
        tc::tmem_ld_wait();
        tc::tc_fence_before_sync();
        __syncwarp();
        if (lane == 0) tc::mbar_arrive_cluster(gu_free);
#pragma unroll
        for (int b = 4 - kAhead; b < 4; ++b) convert(b);
        if (!(ok = wait_bar(&B.h_empty, phase ^ 1, abort_flag))) break;
#pragma unroll
        for (int k = 0; k < 8; ++k)
          tc::st_shared16(h_at + ((k ^ (row_in_cta & 7)) << 4), w[4 * k], w[4 * k + 1], w[4 * k + 2], w[4 * k + 3]);
        tc::fence_proxy_async_smem();
        __syncwarp();
        if (lane == 0) tc::mbar_arrive(&B.h_full);
        if (c == 0) {
          if (t != first && !(ok = take_y())) break;
          y_row0 = next_row0 + warp_row;
          y_rows = next_rows - warp_row;
          fetch(t + step);
        }
      }
    }
    if (ok && first < A.tiles) take_y();
    if (lane == 0) store_box_done();
  } else if (MASKED && warp > kCopyWarp) {
    // ------------------------------------------------------------------------------------ mask
    // a tile's 32 pieces (32 rows x 32 columns, eight quads per lane) are dealt to six warps
    const int drawer = warp < kFirstEpi ? warp - 2 : warp - (kFirstEpi + kResults) + 2;
    const int y_quads = (A.cols + 3) / 4, groups = (A.cols + 31) / 32;
    philox::Stream words(A.mask);
    uint32_t n = 0;
    for (int t = first; t < A.tiles; t += step, ++n) {
      const int32_t row0 = (A.tile_row0 ? A.tile_row0[t] : t * 256) + (int)rank * 128;
      uint32_t* const out = reinterpret_cast<uint32_t*>(gen + kMask + (n & 1) * kMaskBytes);
      if (!wait_bar(B.mask_empty + (n & 1), ((n >> 1) & 1) ^ 1, abort_flag)) break;
      for (int piece = drawer; piece < 4 * groups; piece += kDrawers) {
        const int row = (piece & 3) * 32 + lane, group = piece >> 2;
        const uint64_t q = (uint64_t)(row0 + row) * y_quads + group * 8;
        uint32_t bits = 0u;
#pragma unroll
        for (int part = 0; part < 2; ++part) {
          uint4 w[4];                                      // four quads at a time: a quad is a chain of ten dependent products
#pragma unroll
          for (int k = 0; k < 4; ++k) w[k] = words.quad(A.mask, q + 4 * part + k);       // (past the row's end: words that nothing uses)
#pragma unroll
          for (int k = 0; k < 4; ++k)
            bits |= ((w[k].x > A.mask.lim ? 1u : 0u) | (w[k].y > A.mask.lim ? 2u : 0u) | (w[k].z > A.mask.lim ? 4u : 0u) |
                     (w[k].w > A.mask.lim ? 8u : 0u)) << (16 * part + 4 * k);
        }
        out[group * 128 + row] = bits;
      }
      __syncwarp();
      if (lane == 0) tc::mbar_arrive(B.mask_full + (n & 1));
    }
  }
  // ------------------------------------------------------------------------------------ the end
  if (*abort_flag) {
    if (threadIdx.x == 0) atomicMin(A.status, (int32_t)GNNCO_INTERNAL);
    const long long t0 = clock64();                        // copies and products already issued end before the memory goes
    while (clock64() - t0 < 1000000ll) {}
  }
  tc::tc_fence_before_sync();
  __syncthreads();
  tc::cluster_sync_all();
  if (warp == 0) tc::tmem_dealloc_pair(tmem, 512);
}

}  // namespace

int32_t launch_fused(const Maps& maps, const Args& args, int device, int sms, cudaStream_t st) {
  static std::atomic<int> allowed{0}, allowed_masked{0};
  const int32_t rc = args.masked ? allow_shared_memory(fused_forward<true>, kFusedSmem, device, allowed_masked)
                                 : allow_shared_memory(fused_forward<false>, kFusedSmem, device, allowed);
  if (rc != GNNCO_OK) return rc;
  const int pairs = resident_pairs(device, sms), clusters = args.tiles < pairs ? args.tiles : pairs;
  if (args.masked) return launch_clusters(fused_forward<true>, fused_threads(true), kFusedSmem, maps, args, clusters, 2, st);
  return launch_clusters(fused_forward<false>, fused_threads(false), kFusedSmem, maps, args, clusters, 2, st);
}

}  // namespace ff
