// The gated feed-forward block's backward pass up to dx as ONE kernel, for bfloat16 operands, widths F, F_out <= 128 and F a multiple of 8: dg
// and du are multiplied where they were computed.
//
//   a CTA takes 128 rows of x and dy', which stay in shared memory, and walks H in chunks of 64 columns:
//     G(c)   [g | u] = x [Wg | Wu],  dh = dy' Wd^T      128 x 192 in tensor memory (two buffers)
//     result warps   h, dg, du -> bfloat16, into shared memory, in the layout of an MMA operand, from where they are also
//                    copied to memory: the weight gradients read them
//     D(c)   dx += dg Wg^T + du Wu^T                    128 x F, in tensor memory until the last chunk
//
// G(c + 1) runs while chunk c is converted, across tiles too.  Whichever of the next G and the next D has its operands is issued: D in turn
// with G would wait for weights that take the place of its own (1.13 M x 128 x 256: 667 us, this way 612; two launches 728).  One copy of a
// chunk's weights serves both: G reads Wg and Wu along their rows, D across them.  (A pair of CTAs would have to hold different
// halves for the two.)  A tile's dx is taken out after the first chunk of the next tile.
// What bounds it: 4,500 cycles a chunk, of which a place for weights is held for 6,500 of two chunks from its copy to D, and the 48 KB
// of h, dg and du take 2,900 on their way to memory (without them 500 us).  Two teams of result warps that take chunks in turn
// spilled registers and held the one buffer of h longer: 777 us.
//
// Shared memory: x 32 KB, dy' 32 KB, h, dg and du 48 KB, two chunks of Wg, Wu, Wd 96 KB, staging of dx 16 KB.
// Roles of the warps: 0 products, 1 copies, 2 stores h, dg and du, 4-19 results.
#include "gated_ff_tiles.cuh"

namespace ff {
namespace {

constexpr int kChunk = 64;                                 // columns of h
constexpr uint32_t kXBlock = 16384, kWBlock = 8192;        // 128 or 64 rows of 64 columns
constexpr uint32_t kX = 0, kDy = 2 * kXBlock, kHdd = 4 * kXBlock, kW = kHdd + 3 * kXBlock, kWSlot = 6 * kWBlock, kStaging = kW + 2 * kWSlot;
constexpr uint32_t kWarpStaging = 1024;                    // 32 rows x 16 columns of dx
constexpr uint32_t kBars = kStaging + kEpiWarps * kWarpStaging, kBackSmem = 1024 + kBars + 256;
static_assert(kBackSmem <= 232448, "fits one SM");
constexpr uint32_t kPart = 192, kDxColumn = 384;           // tensor memory: g, u, dh twice; dx

struct Bars {
  uint64_t x_full, x_empty, w_full[2], w_empty[2], part_full[2], part_empty[2], h_full, h_empty, dx_full, dx_empty;
  uint32_t tmem, abort_flag;
};
static_assert(sizeof(Bars) <= 256, "fits");

__global__ void __launch_bounds__(kThreads, 1) fused_backward(const __grid_constant__ Maps maps, const __grid_constant__ CUtensorMap dx_map,
                                                              const __grid_constant__ Args A) {
  extern __shared__ uint8_t smem_raw[];
  const uint32_t sbase = (tc::smem_u32(smem_raw) + 1023u) & ~1023u;
  uint8_t* gen = smem_raw + (sbase - tc::smem_u32(smem_raw));
  Bars& B = *reinterpret_cast<Bars*>(gen + kBars);
  volatile uint32_t* abort_flag = &B.abort_flag;
  asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const int first = blockIdx.x, step = gridDim.x;
  const int x_blocks = (A.cols + 63) >> 6, dy_blocks = (A.K[0] + 63) >> 6;    // of F and F_out: one or two
  const int chunks = (A.K[1] + kChunk - 1) / kChunk;       // of H
  const int tiles_here = first < A.tiles ? (A.tiles - first + step - 1) / step : 0;
  const int32_t total = tiles_here * chunks;

  if (threadIdx.x == 0) {
    tc::mbar_init(&B.x_full, 1);
    tc::mbar_init(&B.x_empty, 1);
    for (int i = 0; i < 2; ++i) {
      tc::mbar_init(B.w_full + i, 1);
      tc::mbar_init(B.w_empty + i, 1);
      tc::mbar_init(B.part_full + i, 1);
      tc::mbar_init(B.part_empty + i, kEpiWarps);
    }
    tc::mbar_init(&B.h_full, kEpiWarps);
    tc::mbar_init(&B.h_empty, 2);                          // multiplied and stored
    tc::mbar_init(&B.dx_full, 1);
    tc::mbar_init(&B.dx_empty, kEpiWarps);
    *abort_flag = 0;
    tc::fence_mbar_init();
  }
  if (warp == 0) tc::tmem_alloc(&B.tmem, 512);
  tc::tc_fence_before_sync();
  __syncthreads();
  tc::tc_fence_after_sync();
  const uint32_t tmem = B.tmem;

  if (warp == kCopyWarp) {
    // -------------------------------------------------------------------------------- operands
    const uint32_t leader = tc::elect_one();
    auto wait = [&](uint64_t* bar, uint32_t parity) { return __all_sync(0xffffffffu, wait_bar(bar, parity, abort_flag)) != 0; };
    Walk<kDown, false, true, true> walk(A, first, step);
    asm volatile("griddepcontrol.wait;" ::: "memory");     // (as in gated_ff_tiles.cuh: everything else hangs on the copies)
    const uint32_t x_bar = tc::smem_u32(&B.x_full);
    uint32_t x_phase = 1;                                  // the first round waits for nothing
    int32_t i = 0;
    bool ok = true;
    while (walk.any() && ok) {
      const Tile T = walk.take();
      for (int c = 0; c < chunks; ++c, ++i) {
        const uint32_t slot = i & 1, bar = tc::smem_u32(B.w_full + slot), at = sbase + kW + slot * kWSlot;
        if (!(ok = wait(B.w_empty + slot, ((uint32_t)i >> 1 & 1) ^ 1))) break;
        expect_bytes<false>(leader, bar, (2 * x_blocks + dy_blocks) * kWBlock);
        for (int k = 0; k < 2; ++k) load_box_of_set<false>(leader, at + k * 2 * kWBlock, &maps.b[k], c * kChunk, 0, T.set, bar);   // all F rows
        for (int kb = 0; kb < dy_blocks; ++kb)
          load_box_of_set<false>(leader, at + (4 + kb) * kWBlock, &maps.b[2], kb * 64, c * kChunk, T.set, bar);
        if (c == 0) {
          if (!(ok = wait(&B.x_empty, x_phase))) break;
          expect_bytes<false>(leader, x_bar, (x_blocks + dy_blocks) * kXBlock);
          for (int kb = 0; kb < x_blocks; ++kb) load_box<false>(leader, sbase + kX + kb * kXBlock, &maps.a[0], kb * 64, T.row0, 0, x_bar);
          for (int kb = 0; kb < dy_blocks; ++kb) load_box<false>(leader, sbase + kDy + kb * kXBlock, &maps.a[1], kb * 64, T.row0, 0, x_bar);
        }
        if (c == 1 % chunks && walk.any()) {
          for (int kb = 0; kb < x_blocks; ++kb) prefetch_box(leader, &maps.a[0], kb * 64, walk.row(), 0);
          for (int kb = 0; kb < dy_blocks; ++kb) prefetch_box(leader, &maps.a[1], kb * 64, walk.row(), 0);
        }
      }
      x_phase ^= 1;
    }
    __syncwarp();
  } else if (warp == kMmaWarp) {
    // -------------------------------------------------------------------------------- products
    if (tc::elect_one()) {
      const uint32_t gu_idesc = tc::idesc_bf16_f32(128, 128, false, true), dh_idesc = tc::idesc_bf16_f32(128, 64, false, false),
                     dx_idesc = tc::idesc_bf16_f32(128, 64 * x_blocks, false, false);
      int gc = 0, dc = 0;                                  // chunk of the tile that G and D are at
      uint32_t x_phase = 0, dx_phase = 1;
      uint32_t i = 0, j = 0;                               // the next G and D
      long long t0 = clock64();
      while (j < (uint32_t)total) {
        bool idle = true;
        if (const uint32_t b = i & 1, phase = i >> 1 & 1;
            i < (uint32_t)total && tc::mbar_test(B.part_empty + b, phase ^ 1) && (gc != 0 || tc::mbar_test(&B.x_full, x_phase)) &&
            tc::mbar_test(B.w_full + b, phase)) {
          idle = false;
          tc::tc_fence_after_sync();
          const uint32_t at = sbase + kW + b * kWSlot, acc = tmem + b * kPart;
          for (int kb = 0; kb < dy_blocks; ++kb) {
            const uint64_t a0 = tc::smem_desc_sw128(sbase + kDy + kb * kXBlock, 16, 1024), b0 = tc::smem_desc_sw128(at + (4 + kb) * kWBlock, 16, 1024);
            const int steps = min(4, (A.K[0] - kb * 64 + 15) >> 4);
#pragma unroll
            for (int k = 0; k < 4; ++k)
              if (k < steps) tc::mma_bf16(acc + 128, a0 + 2 * k, b0 + 2 * k, dh_idesc, kb + k != 0);
          }
          for (int kb = 0; kb < x_blocks; ++kb) {
            const uint64_t a0 = tc::smem_desc_sw128(sbase + kX + kb * kXBlock, 16, 1024), b0 = tc::smem_desc_sw128(at + kb * kWBlock, 2 * kWBlock, 1024);
            const int steps = min(4, (A.cols - kb * 64 + 15) >> 4);
#pragma unroll
            for (int k = 0; k < 4; ++k)
              if (k < steps) tc::mma_bf16(acc, a0 + 2 * k, b0 + 128 * k, gu_idesc, kb + k != 0);
          }
          tc::mma_commit(B.part_full + b);
          if (++gc == chunks) {
            gc = 0;
            x_phase ^= 1;
            tc::mma_commit(&B.x_empty);
          }
          ++i;
        }
        if (j < i && tc::mbar_test(&B.h_full, j & 1) && (dc != 0 || tc::mbar_test(&B.dx_empty, dx_phase))) {
          idle = false;
          const uint32_t at = sbase + kW + (j & 1) * kWSlot;
          if (dc == 0) dx_phase ^= 1;
          tc::tc_fence_after_sync();
          const int steps = min(4, (A.K[1] - dc * kChunk + 15) >> 4);
#pragma unroll
          for (int m = 0; m < 2; ++m) {
            const uint64_t a0 = tc::smem_desc_sw128(sbase + kHdd + (1 + m) * kXBlock, 16, 1024), b0 = tc::smem_desc_sw128(at + m * 2 * kWBlock, 16, 1024);
#pragma unroll
            for (int k = 0; k < 4; ++k)
              if (k < steps) tc::mma_bf16(tmem + kDxColumn, a0 + 2 * k, b0 + 2 * k, dx_idesc, dc + m + k != 0);
          }
          tc::mma_commit(B.w_empty + (j & 1));
          tc::mma_commit(&B.h_empty);
          if (++dc == chunks) {
            dc = 0;
            tc::mma_commit(&B.dx_full);
          }
          ++j;
        }
        if (!idle) t0 = clock64();
        else if (*abort_flag) break;
        else if (clock64() - t0 > 4000000000ll) {
          *abort_flag = 1;
          break;
        }
      }
    }
  } else if (warp == 2) {
    // --------------------------------------------------------------------------------- h, dg, du to memory
    // lanes 0-11: 32 rows of one of the three.  (The ragged end of a subgraph is stored by the result warps: a box would reach into
    // the next one's rows.)
    const int which = lane >> 2, quarter = lane & 3;
    const bool mine = lane < 12 && A.out[0] != nullptr;
    int32_t i = 0;
    bool ok = true;
    for (int t = first; t < A.tiles && ok; t += step) {
      const int32_t row0 = A.tile_row0 ? A.tile_row0[t] : t * 128;
      const int32_t rows = A.tile_row0 ? A.tile_rows[t] : (int32_t)min((int64_t)128, A.rows - (int64_t)t * 128);
      for (int c = 0; c < chunks; ++c, ++i) {
        if (!(ok = __all_sync(0xffffffffu, wait_bar(&B.h_full, i & 1, abort_flag)) != 0)) break;
        if (mine && rows - quarter * 32 >= 32) {
          store_box(&maps.out[which], sbase + kHdd + which * kXBlock + quarter * 4096, c * kChunk, row0 + quarter * 32, 0);
          store_box_read();
        }
        __syncwarp();
        if (lane == 0) tc::mbar_arrive(&B.h_empty);
      }
    }
    store_box_done();
  } else if (warp >= kFirstEpi) {
    // --------------------------------------------------------------------------------- results
    const int quarter = warp & 3, column = (warp - kFirstEpi) >> 2;
    const uint32_t lanes = (uint32_t)(quarter * 32) << 16;
    const int local = quarter * 32 + lane;
    const uint32_t h_at = sbase + kHdd + local * 128, stage_at = sbase + kStaging + (warp - kFirstEpi) * kWarpStaging;
    uint32_t dx_phase = 0;
    // the tile whose dx is still to be taken out: its first row of this warp, how many the tile has from there on
    int32_t dx_row0 = 0, dx_rows = 0;
    bool ok = true;
    auto take_dx = [&] {
      if (!wait_bar(&B.dx_full, dx_phase, abort_flag)) return false;
      dx_phase ^= 1;
      tc::tc_fence_after_sync();
      const int c0 = column * 32;
      const bool in = c0 < A.cols;
      uint32_t w[16];
      if (in) {
        uint32_t r[32];
        tmem_load(tmem + kDxColumn + lanes + c0, r);
        tc::tmem_ld_wait();
#pragma unroll
        for (int k = 0; k < 16; ++k) w[k] = vio::pack_bf16(__uint_as_float(r[2 * k]), __uint_as_float(r[2 * k + 1]));
      }
      tc::tc_fence_before_sync();
      __syncwarp();
      if (lane == 0) tc::mbar_arrive(&B.dx_empty);
      if (!in) return true;
      if (dx_rows >= 32) {
#pragma unroll
        for (int b = 0; b < 2; ++b) {
          if (c0 + 16 * b >= A.cols) break;
          if (lane == 0) store_box_read();                 // the box before has left the tile
          __syncwarp();
          tc::st_shared16(stage_at + lane * 32, w[8 * b], w[8 * b + 1], w[8 * b + 2], w[8 * b + 3]);
          tc::st_shared16(stage_at + lane * 32 + 16, w[8 * b + 4], w[8 * b + 5], w[8 * b + 6], w[8 * b + 7]);
          tc::fence_proxy_async_smem();
          __syncwarp();
          if (lane == 0) store_box(&dx_map, stage_at, c0 + 16 * b, dx_row0, 0);
        }
      } else if (lane < dx_rows) {
        __nv_bfloat16* const to = static_cast<__nv_bfloat16*>(A.y) + (int64_t)(dx_row0 + lane) * A.y_ld + c0;
#pragma unroll
        for (int k = 0; k < 4; ++k)                        // (F is a multiple of 8)
          if (c0 + 8 * k < A.cols) *reinterpret_cast<uint4*>(to + 8 * k) = make_uint4(w[4 * k], w[4 * k + 1], w[4 * k + 2], w[4 * k + 3]);
      }
      return true;
    };
    int32_t next_row0 = 0, next_rows = 0;
    auto fetch = [&](int t) {
      if (t >= A.tiles) return;
      next_row0 = A.tile_row0 ? A.tile_row0[t] : t * 128;
      next_rows = A.tile_row0 ? A.tile_rows[t] : (int32_t)min((int64_t)128, A.rows - (int64_t)t * 128);
    };
    fetch(first);
    int32_t i = 0;
    for (int t = first; t < A.tiles && ok; t += step) {
      const int32_t row0 = next_row0 + quarter * 32, rows_here = next_rows - quarter * 32;
      for (int c = 0; c < chunks; ++c, ++i) {
        const uint32_t b = i & 1;
        if (!(ok = wait_bar(B.part_full + b, (uint32_t)i >> 1 & 1, abort_flag))) break;
        tc::tc_fence_after_sync();
        float f[3][16];
        {
          uint32_t r[3][16];
#pragma unroll
          for (int x = 0; x < 3; ++x) tmem_load(tmem + b * kPart + lanes + 64 * x + 16 * column, r[x]);
          tc::tmem_ld_wait();
#pragma unroll
          for (int x = 0; x < 3; ++x)
#pragma unroll
            for (int e = 0; e < 16; ++e) f[x][e] = __uint_as_float(r[x][e]);
        }
        tc::tc_fence_before_sync();
        __syncwarp();
        if (lane == 0) tc::mbar_arrive(B.part_empty + b);
        if (A.act == GNNCO_SILU) gate<true, GNNCO_SILU>(f, A.scale);
        else if (A.act == GNNCO_GELU) gate<true, GNNCO_GELU>(f, A.scale);
        else gate<true, GNNCO_RELU>(f, A.scale);
        uint32_t w[3][8];
#pragma unroll
        for (int x = 0; x < 3; ++x)
#pragma unroll
          for (int k = 0; k < 8; ++k) w[x][k] = vio::pack_bf16(f[x][2 * k], f[x][2 * k + 1]);
        if (!(ok = wait_bar(&B.h_empty, (i & 1) ^ 1, abort_flag))) break;
#pragma unroll
        for (int x = 0; x < 3; ++x)
#pragma unroll
          for (int k = 0; k < 2; ++k)
            tc::st_shared16(h_at + x * kXBlock + (((2 * column + k) ^ (local & 7)) << 4), w[x][4 * k], w[x][4 * k + 1], w[x][4 * k + 2], w[x][4 * k + 3]);
        tc::fence_proxy_async_smem();
        __syncwarp();
        if (lane == 0) tc::mbar_arrive(&B.h_full);
        const int c0 = c * kChunk + 16 * column;
        if (A.out[0] != nullptr && rows_here < 32 && lane < rows_here && c0 < A.out_ld) {
#pragma unroll
          for (int x = 0; x < 3; ++x) store32(A.out[x] + (int64_t)(row0 + lane) * A.out_ld + c0, w[x]);
        }
        if (c == 0) {
          if (t != first && !(ok = take_dx())) break;
          dx_row0 = row0;
          dx_rows = rows_here;
          fetch(t + step);
        }
      }
    }
    if (ok && first < A.tiles) take_dx();
    if (lane == 0) store_box_done();
  }
  // ------------------------------------------------------------------------------------ the end
  if (*abort_flag) {
    if (threadIdx.x == 0) atomicMin(A.status, (int32_t)GNNCO_INTERNAL);
    const long long t0 = clock64();                        // copies and products already issued end before the memory goes
    while (clock64() - t0 < 1000000ll) {}
  }
  tc::tc_fence_before_sync();
  __syncthreads();
  if (warp == 0) tc::tmem_dealloc(tmem, 512);
}

}  // namespace

int32_t launch_fused_back(const Maps& maps, const CUtensorMap& dx_map, const Args& args, int device, int sms, cudaStream_t st) {
  static std::atomic<int> allowed{0};
  const int32_t rc = allow_shared_memory(fused_backward, kBackSmem, device, allowed);
  if (rc != GNNCO_OK) return rc;
  cudaLaunchConfig_t cfg{};
  cfg.gridDim = dim3(args.tiles < sms ? args.tiles : sms);
  cfg.blockDim = dim3(kThreads);
  cfg.dynamicSmemBytes = kBackSmem;
  cfg.stream = st;
  cudaLaunchAttribute attr[1];
  attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr[0].val.programmaticStreamSerializationAllowed = 1;
  cfg.attrs = attr;
  cfg.numAttrs = args.chained ? 1 : 0;
  GNNCO_CUDA_TRY(cudaLaunchKernelEx(&cfg, fused_backward, maps, dx_map, args));
  return GNNCO_OK;
}

}  // namespace ff
