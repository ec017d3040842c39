// The tiled tensor-core products of the gated feed-forward block (kinds and formulas: gated_ff.cuh).
//
// One persistent CTA per SM, or a cluster of two CTAs that share a tile of 256 rows (tcgen05 .cta_group::2: each CTA stages its
// own 128 rows of A and half of B).  Roles of the twenty warps:
//   warp 0      issues the MMAs (in a pair, the even CTA's)
//   warp 1      issues the TMA copies of this CTA's operands
//   warps 4-19  results: TMEM lanes 32 (w % 4) .., groups of 32 columns (16 of g, u and dh each) in turn.  In bfloat16 two teams of
//               eight take the tiles in turn: a team waits, loads, computes and stores one after the other, so the other one's
//               arithmetic runs meanwhile
// A stage of the ring holds 64 of the contraction: A in the first half, B behind it, each as LIMBS matrices of bfloat16.  Operands
// whose contraction runs along memory (x, dy, h, dg, du as A; Wd, Wg, Wu in the backward products) are k-major boxes of 64
// columns, the others (the weights of the forward products, everything in the weight gradients) n-major boxes of 64 x 64:
// no operand is ever transposed in memory.  Columns past an operand's end are filled with zeros by the copies.  Rows past a
// subgraph's end belong to the next one: their results are not stored, and where rows are what is summed (kWeights) the copying
// warp sets them to zero in shared memory before it announces the stage.
//
// LIMBS = 1 (bfloat16): a tile's products are summed in one of two TMEM buffers of 256 columns, so that the next tile is multiplied
// while this one is converted and stored.
// kGluBack has three accumulators of 128 columns (wide tiles: at 64 columns the copies, not the products, took the time).  Four such
// quarters of TMEM go round: dh of the next tile is summed in the free one while this tile's are converted.
// LIMBS = 3 (float32): a = a1 + a2 + a3 in bfloat16; the six products a_i b_j with i + j <= 4 are summed, what is left out is
// below 2^-24 of the product.  The tensor core cuts off low bits whenever it adds to an accumulator, so sums stay short:
// every stage starts an accumulator of its own (buffers in turn), adds the five small products first and the large one last, and the
// result warps add the stages up in float32 registers, rounded to nearest.
//
// What bounds them and what they took: wide blocks the tensor pipe (65,536 x 1,024 x 2,731 bfloat16, g, u and h at 1.53 PFLOP/s, the
// down product at 1.48; pipe 83 to 88 % active), narrow ones memory and the results' conversion (400,000 x 128 x 256 bfloat16: weight
// gradients 161 us at 5.5 TB/s, dx 86 us at 6.3, h, dg and du 182 us at 4.6 with 48 % of the issue slots; float32 forward 290 and
// 169 us, tensor pipe 67 and 54 %).
//
// The launches of a call are chained by programmatic dependence: a kernel sets itself up while the one before it ends.
// Every wait has a limit; a CTA that gives up raises the handle's status word, skips its work and leaves.
#pragma once

#include "gated_ff.cuh"
#include "tc_common.cuh"
#include "vec_io.cuh"

namespace ff {

constexpr int kMmaWarp = 0, kCopyWarp = 1, kFirstEpi = 4, kEpiWarps = 16, kThreads = 640;
constexpr uint32_t kRing = 196608;                         // 6 stages of 32 KB or 2 of 96 KB
constexpr uint32_t kStageBytes = 32 * 16 * 4;              // a result warp's staging tile: 32 rows x 16 columns
constexpr uint32_t kSmem = 1024 + kRing + kEpiWarps * kStageBytes + 256;
constexpr uint32_t kBuf = 256;                             // TMEM columns of an accumulator buffer
static_assert(kSmem <= 232448, "fits one SM");

// ------------------------------------------------------------------------------------- small pieces
// The whole warp calls these with the same operands and one lane's `leader` != 0: the operands stay in uniform registers.  (Inside an
// `if (lane == 0)` each was moved there per instruction, 150 cycles a copy, and the copying warp could not keep up.)
template <bool PAIR>
__device__ __forceinline__ void load_box(uint32_t leader, uint32_t dst, const CUtensorMap* map, int32_t x, int32_t y, int32_t z, uint32_t bar) {
  if constexpr (PAIR)
    asm volatile("{\n\t.reg .pred go;\n\tsetp.ne.b32 go, %6, 0;\n\t"
                 "@go cp.async.bulk.tensor.3d.cta_group::2.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1, {%2, %3, %4}], [%5];\n\t}"
                 ::"r"(dst), "l"(map), "r"(x), "r"(y), "r"(z), "r"(bar), "r"(leader) : "memory");
  else
    asm volatile("{\n\t.reg .pred go;\n\tsetp.ne.b32 go, %6, 0;\n\t"
                 "@go cp.async.bulk.tensor.3d.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1, {%2, %3, %4}], [%5];\n\t}"
                 ::"r"(dst), "l"(map), "r"(x), "r"(y), "r"(z), "r"(bar), "r"(leader) : "memory");
}
template <bool PAIR>
__device__ __forceinline__ void load_box_of_set(uint32_t leader, uint32_t dst, const CUtensorMap* map, int32_t x, int32_t y, int32_t set, uint32_t bar) {
  if constexpr (PAIR)
    asm volatile("{\n\t.reg .pred go;\n\tsetp.ne.b32 go, %7, 0;\n\t"
                 "@go cp.async.bulk.tensor.4d.cta_group::2.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1, {%2, %3, %4, %5}], [%6];\n\t}"
                 ::"r"(dst), "l"(map), "r"(x), "r"(y), "r"(set), "r"(0), "r"(bar), "r"(leader) : "memory");
  else
    asm volatile("{\n\t.reg .pred go;\n\tsetp.ne.b32 go, %7, 0;\n\t"
                 "@go cp.async.bulk.tensor.4d.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1, {%2, %3, %4, %5}], [%6];\n\t}"
                 ::"r"(dst), "l"(map), "r"(x), "r"(y), "r"(set), "r"(0), "r"(bar), "r"(leader) : "memory");
}
// a box of a later load, into L2
__device__ __forceinline__ void prefetch_box(uint32_t leader, const CUtensorMap* map, int32_t x, int32_t y, int32_t z) {
  asm volatile("{\n\t.reg .pred go;\n\tsetp.ne.b32 go, %4, 0;\n\t@go cp.async.bulk.prefetch.tensor.3d.L2.global.tile [%0, {%1, %2, %3}];\n\t}"
               ::"l"(map), "r"(x), "r"(y), "r"(z), "r"(leader) : "memory");
}
__device__ __forceinline__ void prefetch_map(const CUtensorMap* map) { asm volatile("prefetch.tensormap [%0];" ::"l"(map) : "memory"); }
// announces `bytes` on a barrier of this CTA or, by cluster address, of the pair's even one
template <bool PAIR>
__device__ __forceinline__ void expect_bytes(uint32_t leader, uint32_t bar, uint32_t bytes) {
  if constexpr (PAIR)
    asm volatile("{\n\t.reg .pred go;\n\tsetp.ne.b32 go, %2, 0;\n\t@go mbarrier.arrive.expect_tx.shared::cluster.b64 _, [%0], %1;\n\t}"
                 ::"r"(bar), "r"(bytes), "r"(leader) : "memory");
  else
    asm volatile("{\n\t.reg .pred go;\n\tsetp.ne.b32 go, %2, 0;\n\t@go mbarrier.arrive.expect_tx.shared::cta.b64 _, [%0], %1;\n\t}"
                 ::"r"(bar), "r"(bytes), "r"(leader) : "memory");
}
// CLUSTER: what threads of the other CTA wrote before their arrival is to be seen (copies and products complete through the
// barrier itself, and need no more than the usual wait)
template <bool CLUSTER = false>
__device__ __forceinline__ bool wait_bar(uint64_t* bar, uint32_t parity, volatile uint32_t* abort_flag) {
  auto done = [&] { return CLUSTER ? tc::mbar_try_wait_cluster(bar, parity) : tc::mbar_try_wait(bar, parity); };
  if (done()) return true;
  const long long t0 = clock64();
  while (!done()) {
    if (*abort_flag) return false;
    if (clock64() - t0 > 4000000000ll) {
      *abort_flag = 1;
      return false;
    }
  }
  return true;
}
template <bool PAIR>
__device__ __forceinline__ void multiply(uint32_t d, uint64_t a, uint64_t b, uint32_t idesc, bool accumulate) {
  if (PAIR) tc::mma_bf16_pair(d, a, b, idesc, accumulate);
  else tc::mma_bf16(d, a, b, idesc, accumulate);
}
// everything multiplied so far arrives on this barrier, in both CTAs of a pair
template <bool PAIR>
__device__ __forceinline__ void commit(uint64_t* bar) {
  if (PAIR) tc::mma_commit_pair(bar, 3);
  else tc::mma_commit(bar);
}
__device__ __forceinline__ void store32(void* p, const uint32_t (&w)[8]) {   // 32-byte aligned
  asm volatile("st.global.v8.b32 [%0], {%1, %2, %3, %4, %5, %6, %7, %8};" ::"l"(p), "r"(w[0]), "r"(w[1]), "r"(w[2]), "r"(w[3]),
               "r"(w[4]), "r"(w[5]), "r"(w[6]), "r"(w[7]) : "memory");
}
// W float32 of a row -> LIMBS bfloat16 rows; columns [0, W) of them that lie below `width` (a multiple of 16)
template <int LIMBS, int W>
__device__ __forceinline__ void store_limbs(__nv_bfloat16* to, int64_t limb, int width, const float (&f)[W]) {
#pragma unroll
  for (int half = 0; half < W / 16; ++half) {
    if (half * 16 >= width) break;
    float r[16];
#pragma unroll
    for (int e = 0; e < 16; ++e) r[e] = f[half * 16 + e];
#pragma unroll
    for (int l = 0; l < LIMBS; ++l) {
      uint32_t w[8];
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        w[e] = vio::pack_bf16(r[2 * e], r[2 * e + 1]);
        if (l + 1 < LIMBS) {
          r[2 * e] -= vio::bf_lo(w[e]);                    // exact
          r[2 * e + 1] -= vio::bf_hi(w[e]);
        }
      }
      store32(to + l * limb + half * 16, w);
    }
  }
}
__device__ __forceinline__ void tmem_load(uint32_t at, uint32_t (&r)[32]) { tc::tmem_ld_32x32(at, r); }
__device__ __forceinline__ void tmem_load(uint32_t at, uint32_t (&r)[16]) { tc::tmem_ld_32x16(at, r); }

// Two float32 at a time: one instruction for both halves.
struct Two {
  uint64_t v;
  __device__ __forceinline__ Two() {}
  __device__ __forceinline__ Two(float a, float b) : v(vio::pair_of(a, b)) {}
  __device__ __forceinline__ explicit Two(float a) : v(vio::pair_of(a, a)) {}
  __device__ __forceinline__ void get(float& a, float& b) const { vio::unpair(v, a, b); }
};
__device__ __forceinline__ Two operator*(Two a, Two b) {
  Two d;
  asm("mul.rn.f32x2 %0, %1, %2;" : "=l"(d.v) : "l"(a.v), "l"(b.v));
  return d;
}
__device__ __forceinline__ Two operator+(Two a, Two b) {
  Two d;
  asm("add.rn.f32x2 %0, %1, %2;" : "=l"(d.v) : "l"(a.v), "l"(b.v));
  return d;
}
__device__ __forceinline__ Two fma(Two a, Two b, Two c) {
  Two d;
  asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(d.v) : "l"(a.v), "l"(b.v), "l"(c.v));
  return d;
}
// the hardware's 2^x (2 units of 2^-23) and 1 / x (1 unit), results and arguments below 2^-126 as zeros: no range handling around
// them.  (1 / x by a Newton and a third-order step on the arithmetic pipes halves the transcendental instructions, but its nine
// instructions more per pair took the same time alone and more beside the drawing of masks: 2.5 M x 256 x 512 bfloat16 1,588 and,
// with dropout, 2,164 us; this way 1,576 and 1,956.)
__device__ __forceinline__ Two exp2(Two x) {
  float a, b;
  x.get(a, b);
  asm("ex2.approx.ftz.f32 %0, %0;" : "+f"(a));
  asm("ex2.approx.ftz.f32 %0, %0;" : "+f"(b));
  return Two(a, b);
}
__device__ __forceinline__ Two inverse(Two x) {
  float a, b;
  x.get(a, b);
  asm("rcp.approx.ftz.f32 %0, %0;" : "+f"(a));
  asm("rcp.approx.ftz.f32 %0, %0;" : "+f"(b));
  return Two(a, b);
}

// a = act(g) and, for the backward pass, slope = act'(g).
//   SiLU   s = 1 / (1 + 2^(-g log2 e)):  a = g s,  a' = s + a (1 - s)
//   GELU   E = exp(-g^2 / 2), Phi(-|g|) = E t P(t) with t = 1 / (1 + 0.3 |g| / sqrt 2), P of degree 8 fitted to
//          erfc(z) exp(z^2) / (2 t) over t (4.5e-8 of the value at most up to |g| = 14, where Phi is 8e-45; with E and the rest in
//          float32, of a 4.8e-7 up to |g| = 2, 1.5e-6 up to 5 and 7.5e-6 up to 12, where Phi is 2e-33):  a = g Phi(g),  a' = Phi(g) + g E / sqrt(2 pi)
template <int ACT, bool BACK>
__device__ __forceinline__ void activate(Two g, Two& a, Two& slope) {
  if (ACT == GNNCO_SILU) {
    const Two s = inverse(exp2(g * Two(-1.44269504f)) + Two(1.0f));
    a = g * s;
    if (BACK) slope = fma(a, fma(s, Two(-1.0f), Two(1.0f)), s);
  } else if (ACT == GNNCO_GELU) {
    float g0, g1, q0, q1;
    g.get(g0, g1);
    const Two E = exp2(g * g * Two(-0.72134752f));
    const Two t = inverse(fma(Two(fabsf(g0), fabsf(g1)), Two(0.21213203f), Two(1.0f)));
    Two P = fma(t, Two(-0.06476137787103653f), Two(0.24278123676776886f));
    P = fma(t, P, Two(-0.25613829493522644f));
    P = fma(t, P, Two(0.2738591432571411f));
    P = fma(t, P, Two(-0.0473247766494751f));
    P = fma(t, P, Two(0.10746278613805771f));
    P = fma(t, P, Two(0.07416965067386627f));
    P = fma(t, P, Two(0.08535760641098022f));
    P = fma(t, P, Two(0.0845940038561821f));
    (E * t * P).get(q0, q1);
    const Two phi(g0 > 0.0f ? 1.0f - q0 : q0, g1 > 0.0f ? 1.0f - q1 : q1);
    a = g * phi;
    if (BACK) slope = fma(g * Two(0.39894228f), E, phi);
  } else {
    float g0, g1;
    g.get(g0, g1);
    a = Two(g0 > 0.0f ? g0 : (g0 != g0 ? g0 : 0.0f), g1 > 0.0f ? g1 : (g1 != g1 ? g1 : 0.0f));
    if (BACK) slope = Two(g0 > 0.0f ? 1.0f : 0.0f, g1 > 0.0f ? 1.0f : 0.0f);
  }
}
// g, u (and dh) -> h (and dg, du), in place.  One activation for the whole loop: a branch per element would take the elements one after
// the other, each waiting for its exponential (1.28 G elements in 3.4 ms).
template <bool BACK, int ACT, int TENSORS, int W>
__device__ __forceinline__ void gate(float (&f)[TENSORS][W], float scale) {
#pragma unroll
  for (int e = 0; e < W; e += 2) {
    const Two u(f[1][e], f[1][e + 1]);
    Two a, slope;
    activate<ACT, BACK>(Two(f[0][e], f[0][e + 1]), a, slope);
    (a * u).get(f[0][e], f[0][e + 1]);
    if (BACK) {
      const Two dh = Two(f[TENSORS - 1][e], f[TENSORS - 1][e + 1]) * Two(scale);
      (dh * u * slope).get(f[1][e], f[1][e + 1]);
      (dh * a).get(f[TENSORS - 1][e], f[TENSORS - 1][e + 1]);
    }
  }
}
// A box from a result warp's staging tile (2 KB) to columns x .., rows y .. and limb z of a result.  A lane that stored its row by
// itself would send 32 pieces of 32 rows per instruction: for float32 results that took longer than the products.
__device__ __forceinline__ void store_box(const CUtensorMap* map, uint32_t from, int32_t x, int32_t y, int32_t z) {
  asm volatile("cp.async.bulk.tensor.3d.global.shared::cta.bulk_group [%0, {%1, %2, %3}], [%4];" ::"l"(map), "r"(x), "r"(y), "r"(z), "r"(from) : "memory");
  asm volatile("cp.async.bulk.commit_group;" ::: "memory");
}
// all boxes but the last LATER have been read from shared memory
template <int LATER = 0>
__device__ __forceinline__ void store_box_read() { asm volatile("cp.async.bulk.wait_group.read %0;" ::"n"(LATER) : "memory"); }
__device__ __forceinline__ void store_box_done() { asm volatile("cp.async.bulk.wait_group 0;" ::: "memory"); }
// Rows of 64 bytes (16 words of this lane's row), in units of 16 bytes swizzled by bits 1 and 2 of the row; whole warp
__device__ __forceinline__ void stage_row(const CUtensorMap* map, uint32_t stage, int lane, int32_t x, int32_t y, int32_t z, const uint32_t (&w)[16]) {
  if (lane == 0) store_box_read();                         // the box before has left the tile
  __syncwarp();
#pragma unroll
  for (int q = 0; q < 4; ++q)
    tc::st_shared16(stage + lane * 64 + ((q ^ ((lane >> 1) & 3)) << 4), w[4 * q], w[4 * q + 1], w[4 * q + 2], w[4 * q + 3]);
  tc::fence_proxy_async_smem();
  __syncwarp();
  if (lane == 0) store_box(map, stage, x, y, z);
}
// 32 values of this lane's row as LIMBS bfloat16
template <int LIMBS>
__device__ __forceinline__ void stage_limbs(const CUtensorMap* map, uint32_t stage, int lane, int32_t x, int32_t y, float (&f)[32]) {
#pragma unroll
  for (int l = 0; l < LIMBS; ++l) {
    uint32_t w[16];
#pragma unroll
    for (int e = 0; e < 16; ++e) {
      w[e] = vio::pack_bf16(f[2 * e], f[2 * e + 1]);
      if (l + 1 < LIMBS) {
        f[2 * e] -= vio::bf_lo(w[e]);                      // exact
        f[2 * e + 1] -= vio::bf_hi(w[e]);
      }
    }
    stage_row(map, stage, lane, x, y, l, w);
  }
}
// 16 values of this lane's row as LIMBS bfloat16: rows of 32 bytes, in the halves of the tile in turn
template <int LIMBS>
__device__ __forceinline__ void stage_limbs(const CUtensorMap* map, uint32_t stage, int lane, int32_t x, int32_t y, float (&f)[16], uint32_t& turn) {
#pragma unroll
  for (int l = 0; l < LIMBS; ++l) {
    uint32_t w[8];
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      w[e] = vio::pack_bf16(f[2 * e], f[2 * e + 1]);
      if (l + 1 < LIMBS) {
        f[2 * e] -= vio::bf_lo(w[e]);                      // exact
        f[2 * e + 1] -= vio::bf_hi(w[e]);
      }
    }
    if (lane == 0) store_box_read<1>();
    __syncwarp();
    const uint32_t at = stage + turn * 1024;
    tc::st_shared16(at + lane * 32, w[0], w[1], w[2], w[3]);
    tc::st_shared16(at + lane * 32 + 16, w[4], w[5], w[6], w[7]);
    tc::fence_proxy_async_smem();
    __syncwarp();
    if (lane == 0) store_box(map, at, x, y, l);
    turn ^= 1;
  }
}
// 32 values of this lane's row as float32: two boxes of 16 columns
__device__ __forceinline__ void stage_floats(const CUtensorMap* map, uint32_t stage, int lane, int32_t x, int32_t y, const float (&f)[32]) {
#pragma unroll
  for (int b = 0; b < 2; ++b) {
    uint32_t w[16];
#pragma unroll
    for (int e = 0; e < 16; ++e) w[e] = __float_as_uint(f[16 * b + e]);
    stage_row(map, stage, lane, x + 16 * b, y, 0, w);
  }
}

// 32 values of this lane's row (row0 + lane, if that is below rows_here) to out[row][c0 ..], for rows that start anywhere or end inside
// the group: through the staging tile, 16 columns at a time, so that half a warp holds neighbouring columns (column c of row r
// stands at c ^ (r % 16): no bank twice in a read, twice in a write).  Whole warp.
template <bool WIDE>
__device__ __forceinline__ void store_rows(float* stage, int lane, int rows_here, int64_t row0, int c0, int cols, void* out, int64_t ld,
                                           const float (&f)[32]) {
#pragma unroll
  for (int b = 0; b < 2; ++b) {
    if (lane == 0) store_box_read();                       // a box before may still be read from the tile
    __syncwarp();
#pragma unroll
    for (int e = 0; e < 16; ++e) stage[lane * 16 + (e ^ (lane & 15))] = f[16 * b + e];
    __syncwarp();
    const int col = c0 + 16 * b + (lane & 15);
    if (col >= cols) continue;
    for (int r = lane >> 4; r < min(32, rows_here); r += 2) {
      const float x = stage[r * 16 + ((lane & 15) ^ (r & 15))];
      const int64_t to = (row0 + r) * ld + col;
      if (WIDE) static_cast<float*>(out)[to] = x;
      else static_cast<__nv_bfloat16*>(out)[to] = __float2bfloat16_rn(x);
    }
  }
  __syncwarp();
}

struct Tile {
  int32_t row0, rows, n0, m0, problem, slot, set;
  int32_t stages;                                          // of the first contraction
};
// The tiles of a CTA, t = first, first + step ..  They are numbered with the columns fastest, so that CTAs that work at the same time
// share rows.  A short tile takes some 2,000 cycles, so the way from its number to its rows is kept off them: no divisions (the tile of
// rows and of columns advance by a fixed step each), and the entries of the tables are requested one tile ahead, the set, which
// hangs on the row, in the tile before.
template <int KIND, bool PAIR, bool SETS, bool UNIFORM>
class Walk {
  const Args& A;
  int32_t t, step, m, n, dm, dn;
  int32_t a = 0, b = 0, c = 0;                             // table entries of tile t
  int32_t a1 = 0, b1 = 0, set = 0;                         // SETS: (a, b) of the tile after t, the set of t
  bool table;

  // the same value in a uniform register (every lane of the warp holds it)
  static __device__ __forceinline__ int32_t uniform(int32_t v) { return UNIFORM ? __shfl_sync(0xffffffffu, v, 0) : v; }
  __device__ __forceinline__ void advance() {
    t += step;
    m += dm;
    n += dn;
    if (KIND != kWeights && n >= A.n_tiles) {
      n -= A.n_tiles;
      ++m;
    }
  }
  __device__ __forceinline__ void fetch(int32_t& row0, int32_t& rows) {
    if (!table || t >= A.tiles) return;
    if (KIND == kWeights) {
      const int32_t chunk = t / A.per_chunk;
      row0 = A.chunk_begin[chunk];
      rows = A.chunk_end[chunk];
      c = A.chunk_slot[chunk];
    } else {
      row0 = A.tile_row0[m];
      rows = A.tile_rows[m];
    }
  }

 public:
  __device__ __forceinline__ Walk(const Args& args, int first, int by) : A(args), t(first), step(by) {
    table = KIND == kWeights ? A.chunk_begin != nullptr : A.tile_row0 != nullptr;
    if (KIND != kWeights) {
      m = t / A.n_tiles;
      n = t - m * A.n_tiles;
      dm = step / A.n_tiles;
      dn = step - dm * A.n_tiles;
    } else {
      m = n = dm = dn = 0;
    }
    fetch(a, b);
    if (SETS && table && t < A.tiles) {
      set = A.node_part[a];
      const int32_t m0 = m, n0 = n;
      advance();
      fetch(a1, b1);
      t -= step;
      m = m0;
      n = n0;
    }
  }
  __device__ __forceinline__ bool any() const { return t < A.tiles; }
  // this tile, and on to the next
  __device__ __forceinline__ Tile take() {
    constexpr int TM = PAIR ? 256 : 128;
    Tile T;
    if constexpr (KIND == kWeights) {
      const int32_t chunk = t / A.per_chunk;
      int rest = t - chunk * A.per_chunk, q = 0;
      while (rest >= A.p[q].m_tiles * A.p[q].n_tiles) {
        rest -= A.p[q].m_tiles * A.p[q].n_tiles;
        ++q;
      }
      T.problem = uniform(q);
      T.m0 = uniform((rest / A.p[q].n_tiles) * TM);
      T.n0 = uniform((rest % A.p[q].n_tiles) * A.p[q].nt);
      if (table) {
        T.row0 = uniform(a);
        T.rows = uniform(b - a);
        T.slot = uniform(c);
      } else {
        T.row0 = uniform(chunk * A.chunk_rows);
        T.rows = uniform((int32_t)min((int64_t)A.chunk_rows, A.rows - (int64_t)chunk * A.chunk_rows));
        T.slot = A.chunks == 1 ? -1 : uniform(chunk);
      }
      T.set = T.slot < 0 ? -(T.slot + 1) : 0;
      T.stages = (T.rows + 63) >> 6;
      advance();
      fetch(a, b);
    } else {
      T.m0 = T.problem = T.slot = 0;
      T.n0 = uniform(n * A.nt);
      T.row0 = uniform(table ? a : m * TM);
      T.rows = uniform(table ? b : (int32_t)min((int64_t)TM, A.rows - (int64_t)m * TM));
      T.set = SETS ? uniform(set) : 0;
      T.stages = (A.K[0] + 63) >> 6;
      advance();
      if (SETS) {
        a = a1;
        b = b1;
        if (table && any()) set = A.node_part[a];
        const int32_t m0 = m, n0 = n;
        advance();
        fetch(a1, b1);
        t -= step;
        m = m0;
        n = n0;
      } else {
        fetch(a, b);
      }
    }
    return T;
  }
  // the first row of that tile
  __device__ __forceinline__ int32_t row() const { return table ? a : m * (PAIR ? 256 : 128); }
  // a tile whose rows do not matter
  __device__ __forceinline__ void skip() { t += step; }
};

// ------------------------------------------------------------------------------------------- kernel
template <int KIND, int LIMBS, bool PAIR>
__global__ void __launch_bounds__(kThreads, 1) tiles(const __grid_constant__ Maps maps, const __grid_constant__ Args A) {
  constexpr uint32_t kSlot = 32768 * LIMBS, kA = 16384 * LIMBS;
  constexpr int kSlots = kRing / kSlot;
  constexpr uint32_t kBlock = 8192 * LIMBS;                // 64 x 64 of an n-major operand, all limbs
  constexpr int kCtas = PAIR ? 2 : 1;
  constexpr bool kAlongRows = KIND == kWeights;
  constexpr int kSegments = KIND == kGluBack ? 2 : 1;      // contractions one after the other (kDx takes a stage of each in turn)
  constexpr bool kSums = LIMBS > 1;                        // stages are added up in registers
  constexpr bool kQuarters = KIND == kGluBack && !kSums;   // accumulators take quarters of TMEM in turn
  constexpr int kTeams = LIMBS == 1 && !kAlongRows && !kQuarters ? 2 : 1;    // of result warps, tiles in turn
  constexpr int kColumns = kEpiWarps / 4 / kTeams;         // warps of a team that share TMEM lanes

  extern __shared__ uint8_t smem_raw[];
  const uint32_t sbase = (tc::smem_u32(smem_raw) + 1023u) & ~1023u;
  uint8_t* gen = smem_raw + (sbase - tc::smem_u32(smem_raw));
  uint64_t* full = reinterpret_cast<uint64_t*>(gen + kRing + kEpiWarps * kStageBytes);   // the even CTA's is used
  uint64_t* empty = full + kSlots;                         // every CTA's own
  uint64_t* acc_full = empty + kSlots;                     // [2] every CTA's own
  uint64_t* acc_empty = acc_full + 2;                      // [2] the even CTA's is used
  uint64_t* tail = acc_empty + 2;                          // this CTA's stages with rows to be cleared
  uint32_t* tmem_slot = reinterpret_cast<uint32_t*>(tail + 1);
  volatile uint32_t* abort_flag = tmem_slot + 1;
  asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const uint32_t rank = PAIR ? tc::cluster_ctarank() : 0u;
  const int first = blockIdx.x / kCtas, step = gridDim.x / kCtas;

  constexpr int kMapsA = KIND == kWeights ? 3 : KIND == kDx || KIND == kGluBack ? 2 : 1;
  constexpr int kMapsB = KIND == kWeights || KIND == kGluBack ? 3 : KIND == kDown ? 1 : 2;
  if (warp == kCopyWarp && lane < kMapsA + kMapsB) prefetch_map(lane < kMapsA ? &maps.a[lane] : &maps.b[lane - kMapsA]);
  if (threadIdx.x == 0) {
    for (int i = 0; i < kSlots; ++i) {
      tc::mbar_init(full + i, kCtas);
      tc::mbar_init(empty + i, 1);
    }
    for (int i = 0; i < 2; ++i) {
      tc::mbar_init(acc_full + i, 1);
      tc::mbar_init(acc_empty + i, kCtas * kEpiWarps / kTeams);
    }
    tc::mbar_init(tail, 1);
    *abort_flag = 0;
    tc::fence_mbar_init();
  }
  if (warp == 0) {
    if (PAIR) tc::tmem_alloc_pair(tmem_slot, 512);
    else tc::tmem_alloc(tmem_slot, 512);
  }
  tc::tc_fence_before_sync();
  __syncthreads();
  if (PAIR) tc::cluster_sync_all();
  tc::tc_fence_after_sync();
  const uint32_t tmem = *tmem_slot;
  const int more = kAlongRows ? 0 : (A.K[1] + 63) >> 6;    // stages of the second contraction

  if (warp == kCopyWarp) {
    // -------------------------------------------------------------------------------- operands
    const uint32_t leader = tc::elect_one();
    const int rank_u = __shfl_sync(0xffffffffu, (int)rank, 0);
    int tails = 0, slot = 0;
    uint32_t phase = 1;                                    // of `empty`: the first round waits for nothing
    bool ok = true;
    Walk<KIND, PAIR, !kAlongRows, true> walk(A, first, step);
    // The operands are complete from here on.  (The other warps' work hangs on the copies, the results they write included, and the
    // tables are older than the launch before this one.)
    asm volatile("griddepcontrol.wait;" ::: "memory");
    while (walk.any() && ok) {
      const Tile T = walk.take();
      const int set = T.set;
      const int nt = kAlongRows ? A.p[T.problem].nt : A.nt;
      for (int seg = 0; seg < kSegments && ok; ++seg) {
        const bool twin = KIND == kGlu || (KIND == kGluBack && seg == 1);
        const uint32_t bytes = kA + (twin ? 2 : 1) * (nt / kCtas) * 128 * LIMBS;
        const int stages = KIND == kDx ? 2 * T.stages : seg == 0 ? T.stages : more;
        for (int s = 0; s < stages; ++s) {
          const int kb = KIND == kDx ? s >> 1 : s;
          if (!(ok = __all_sync(0xffffffffu, wait_bar(empty + slot, phase, abort_flag)) != 0)) break;
          const uint32_t at = sbase + slot * kSlot, bt = at + kA;
          const uint32_t announce = PAIR ? tc::map_to_cta(tc::smem_u32(full + slot), 0) : tc::smem_u32(full + slot);
          const int valid = kAlongRows ? min(64, T.rows - kb * 64) : 64;
          const uint32_t bar = valid == 64 ? announce : tc::smem_u32(tail);
          expect_bytes<PAIR>(leader, bar, bytes);
          if constexpr (kAlongRows) {
            const int32_t r = (int32_t)T.row0 + kb * 64, m = T.m0 + rank_u * 128, n = T.n0 + rank_u * (nt / kCtas);
            load_box<PAIR>(leader, at, &maps.a[T.problem], m, r, 0, bar);
            load_box<PAIR>(leader, at + kBlock, &maps.a[T.problem], m + 64, r, 0, bar);
            for (int i = 0; i < nt / kCtas / 64; ++i) load_box<PAIR>(leader, bt + i * kBlock, &maps.b[T.problem], n + 64 * i, r, 0, bar);
          } else {
            load_box<PAIR>(leader, at, &maps.a[KIND == kDx ? s & 1 : seg], kb * 64, (int32_t)T.row0 + rank_u * 128, 0, bar);
            if (twin && kQuarters) {
              // 64 gate columns, then the same up columns; in a pair each CTA holds half of both
              load_box_of_set<PAIR>(leader, bt, &maps.b[0], T.n0 + rank_u * 64, kb * 64, set, bar);
              load_box_of_set<PAIR>(leader, bt + kBlock, &maps.b[1], T.n0 + rank_u * 64, kb * 64, set, bar);
            } else if (twin) {
              // gate columns, then up columns; in a pair the even CTA holds the gate's, the odd one the other's
              const int per = nt / 64;
              for (int i = 0; i < 2 * per / kCtas; ++i) {
                const int which = PAIR ? rank_u : i / per, block = PAIR ? i : i % per;
                load_box_of_set<PAIR>(leader, bt + i * kBlock, &maps.b[which], T.n0 + 64 * block, kb * 64, set, bar);
              }
            } else if (KIND == kDown) {
              const int n = T.n0 + rank_u * (nt / kCtas);
              for (int i = 0; i < nt / kCtas / 64; ++i) load_box_of_set<PAIR>(leader, bt + i * kBlock, &maps.b[0], n + 64 * i, kb * 64, set, bar);
            } else {
              load_box_of_set<PAIR>(leader, bt, &maps.b[KIND == kGluBack ? 2 : s & 1], kb * 64, T.n0 + rank_u * (nt / kCtas), set, bar);
            }
          }
          if constexpr (kAlongRows) if (valid < 64) {
            // row k of a 64-column block is 128 bytes at 128 k, whatever the swizzle does inside it; the products take 16 rows at a time
            if (!(ok = __all_sync(0xffffffffu, wait_bar(tail, tails & 1, abort_flag)) != 0)) break;
            ++tails;
            const uint32_t end = at + (2 + nt / kCtas / 64) * kBlock;
            for (uint32_t block = at; block < end; block += 8192)
              for (int b = valid * 128 + lane * 16; b < ((valid + 15) & ~15) * 128; b += 512) tc::st_shared_zero16(block + b);
            tc::fence_proxy_async_smem();
            __syncwarp();
            if (lane == 0) {
              if (PAIR) tc::mbar_arrive_release_cluster(announce);
              else tc::mbar_arrive(full + slot);
            }
          }
          if (++slot == kSlots) {
            slot = 0;
            phase ^= 1;
          }
        }
      }
    }
    __syncwarp();
  } else if (warp == kMmaWarp) {
    // -------------------------------------------------------------------------------- products
    if (rank == 0 && tc::elect_one()) {                    // one thread
      constexpr int M = PAIR ? 256 : 128;
      int slot = 0, part = 0;
      uint32_t phase = 0;
      bool ok = true;
      Walk<KIND, PAIR, false, false> walk(A, first, step);
      while (walk.any() && ok) {
        Tile T = {};
        if (kAlongRows) {
          T = walk.take();
        } else {                                           // every tile is the same here
          T.stages = (A.K[0] + 63) >> 6;
          walk.skip();
        }
        const int nt = kAlongRows ? A.p[T.problem].nt : A.nt;
        bool open = false;                                 // the current part has its buffer
        for (int seg = 0; seg < kSegments && ok; ++seg) {
          const bool twin = KIND == kGlu || (KIND == kGluBack && seg == 1);
          const bool b_n_major = twin || KIND == kDown || KIND == kWeights;
          const int N = twin && !kQuarters ? 2 * nt : nt;
          const uint32_t idesc = tc::idesc_bf16_f32(M, N, kAlongRows, b_n_major);
          if (kQuarters && seg == 1) {
            // g and u take the quarters that dh and g of the tile before held
            if (part >= 1) ok = wait_bar(acc_empty + ((part - 1) & 1), ((part - 1) >> 1) & 1, abort_flag);
            tc::tc_fence_after_sync();
            if (!ok) break;
          }
          const uint32_t b_limb = b_n_major ? 8192 : (uint32_t)(nt / kCtas) * 128;
          const int K = kAlongRows ? T.rows : A.K[seg];
          const int stages = KIND == kDx ? 2 * T.stages : seg == 0 ? T.stages : more;
          for (int s = 0; s < stages; ++s) {
            const int kb = KIND == kDx ? s >> 1 : s;
            if (!open) {
              if (part >= 2 && !kQuarters) ok = wait_bar(acc_empty + (part & 1), ((part >> 1) - 1) & 1, abort_flag);
              tc::tc_fence_after_sync();
              if (!ok) break;
              open = true;
            }
            const uint32_t acc = tmem + (kQuarters ? ((3 * part + seg) & 3) * 128 : (part & 1) * kBuf);
            ok = wait_bar<PAIR && kAlongRows>(full + slot, phase, abort_flag);
            tc::tc_fence_after_sync();
            if (!ok) break;
            const uint32_t at = sbase + slot * kSlot, bt = at + kA;
            const int steps = min(4, (K - kb * 64 + 15) >> 4);       // what lies behind K is zero
            const uint64_t a0 = tc::smem_desc_sw128(at, kAlongRows ? kBlock : 16, 1024);
            const uint64_t b0 = tc::smem_desc_sw128(bt, b_n_major ? kBlock : 16, 1024);
            constexpr uint64_t a_step = kAlongRows ? 128 : 2, a_limb = (kAlongRows ? 8192 : 16384) / 16;
            const uint64_t b_step = b_n_major ? 128 : 2;
            if constexpr (LIMBS == 1) {
#pragma unroll
              for (int k = 0; k < 4; ++k)
                if (k < steps) multiply<PAIR>(acc, a0 + a_step * k, b0 + b_step * k, idesc, s + k != 0);
              if (kQuarters && seg == 1) {
                const uint32_t acc2 = tmem + ((3 * part + 2) & 3) * 128;
#pragma unroll
                for (int k = 0; k < 4; ++k)
                  if (k < steps) multiply<PAIR>(acc2, a0 + a_step * k, b0 + kBlock / 16 + b_step * k, idesc, kb + k != 0);
              }
            } else {
              // a1 b3, a2 b2, a3 b1, a1 b2, a2 b1, then a1 b1
#pragma unroll
              for (int q = 0; q < 6; ++q) {
                const int i = q == 1 || q == 4 ? 1 : q == 2 ? 2 : 0, j = q == 0 ? 2 : q == 1 || q == 3 ? 1 : 0;
                const uint64_t a = a0 + i * a_limb, b = b0 + (uint64_t)(j * b_limb / 16);
#pragma unroll
                for (int k = 0; k < 4; ++k)
                  if (k < steps) multiply<PAIR>(acc, a + a_step * k, b + b_step * k, idesc, q + k != 0);
              }
            }
            commit<PAIR>(empty + slot);
            if (kSums) {
              commit<PAIR>(acc_full + (part & 1));
              ++part;
              open = false;
            }
            if (++slot == kSlots) {
              slot = 0;
              phase ^= 1;
            }
          }
        }
        if (!kSums && ok && open) {
          commit<PAIR>(acc_full + (part & 1));
          ++part;
        }
      }
    }
  } else if (warp >= kFirstEpi) {
    // --------------------------------------------------------------------------------- results
    const int quarter = warp & 3, column = ((warp - kFirstEpi) >> 2) % kColumns, team = ((warp - kFirstEpi) >> 2) / kColumns;
    const uint32_t lanes = (uint32_t)(quarter * 32) << 16;
    const uint32_t free_bar = PAIR ? tc::map_to_cta(tc::smem_u32(acc_empty), 0) : tc::smem_u32(acc_empty);
    float* const stage = reinterpret_cast<float*>(gen + kRing + (warp - kFirstEpi) * kStageBytes);
    const uint32_t stage_at = sbase + kRing + (warp - kFirstEpi) * kStageBytes;
    constexpr int kW = KIND == kGluBack ? 16 : 32;         // columns of a group
    constexpr int kGroups = (KIND == kGlu || (KIND == kGluBack && kSums) ? 4 : 8) / kColumns;      // groups of a warp, at most
    constexpr int kTensors = KIND == kGlu ? 2 : KIND == kGluBack ? 3 : 1;
    float v[kSums ? kGroups : 1][kTensors][kW];
    int part = team;
    uint32_t turn = 0;                                     // half of the staging tile
    bool ok = true;
    auto release = [&]() {
      tc::tc_fence_before_sync();
      __syncwarp();
      if (lane == 0) {
        if (PAIR) tc::mbar_arrive_cluster(free_bar + (part & 1) * 8);
        else tc::mbar_arrive(acc_empty + (part & 1));
      }
      part += kTeams;
    };
    philox::Stream words(A.mask);
    Walk<KIND, PAIR, false, false> walk(A, first + team * step, kTeams * step);
    while (walk.any() && ok) {
      const Tile T = walk.take();
      const int nt = kAlongRows ? A.p[T.problem].nt : A.nt;
      const int cols = kAlongRows ? A.p[T.problem].N : A.cols;
      const int groups = min(nt, cols - T.n0 + kW - 1) / kW;         // that hold columns of the result
      const int local = (int)rank * 128 + quarter * 32 + lane;
      const int stages = T.stages + more;
      if (kSums) {
#pragma unroll
        for (int i = 0; i < kGroups; ++i)
#pragma unroll
          for (int x = 0; x < kTensors; ++x)
#pragma unroll
            for (int e = 0; e < kW; ++e) v[kSums ? i : 0][x][e] = 0.0f;
        for (int kb = 0; kb < stages && ok; ++kb) {
          if (!wait_bar(acc_full + (part & 1), (part >> 1) & 1, abort_flag)) { ok = false; break; }
          tc::tc_fence_after_sync();
          const uint32_t acc = tmem + lanes + (part & 1) * kBuf;
          const bool second = kb >= T.stages;                // of g, u and dh, the stages of dh come first
#pragma unroll
          for (int i = 0; i < kGroups; ++i) {
            const int c = column + kColumns * i;
            if (c >= groups) continue;
#pragma unroll
            for (int x = 0; x < kTensors; ++x) {
              if (KIND == kGluBack && second == (x == 2)) continue;
#pragma unroll
              for (int b = 0; b < kW / 16; ++b) {
                uint32_t r[16];
                tmem_load(acc + (x == 1 ? nt : 0) + c * kW + 16 * b, r);
                tc::tmem_ld_wait();
#pragma unroll
                for (int e = 0; e < 16; ++e) v[kSums ? i : 0][x][16 * b + e] += __uint_as_float(r[e]);
              }
            }
          }
          release();
        }
      } else if (stages > 0) {
        if (!wait_bar(acc_full + (part & 1), (part >> 1) & 1, abort_flag)) { ok = false; break; }
        tc::tc_fence_after_sync();
      }
      if (!ok) break;
      const uint32_t acc = tmem + lanes + (part & 1) * kBuf;
      bool holding = !kSums && stages > 0;                 // the accumulators: given back once this warp's are in registers
      if (holding && column >= groups) {
        release();
        holding = false;
      }
#pragma unroll
      for (int i = 0; i < kGroups; ++i) {
        const int c = column + kColumns * i;
        if (c >= groups) continue;
        float (&f)[kTensors][kW] = v[kSums ? i : 0];
        if (!kSums) {
          if (stages > 0) {
            uint32_t r[kTensors][kW];
#pragma unroll
            for (int x = 0; x < kTensors; ++x)
              tmem_load(kQuarters ? tmem + lanes + ((3 * part + (x + 1) % 3) & 3) * 128 + c * kW : acc + x * nt + c * kW, r[x]);
            tc::tmem_ld_wait();
#pragma unroll
            for (int x = 0; x < kTensors; ++x)
#pragma unroll
              for (int e = 0; e < kW; ++e) f[x][e] = __uint_as_float(r[x][e]);
            if (holding && (i + 1 == kGroups || c + kColumns >= groups)) {
              release();
              holding = false;
            }
          } else {
#pragma unroll
            for (int x = 0; x < kTensors; ++x)
#pragma unroll
              for (int e = 0; e < kW; ++e) f[x][e] = 0.0f;
          }
        }
        const int c0 = T.n0 + c * kW;
        if constexpr (KIND == kGlu || KIND == kGluBack) {
          constexpr bool kBack = KIND == kGluBack;
          if (A.act == GNNCO_SILU) gate<kBack, GNNCO_SILU>(f, A.scale);
          else if (A.act == GNNCO_GELU) gate<kBack, GNNCO_GELU>(f, A.scale);
          else gate<kBack, GNNCO_RELU>(f, A.scale);
          const int rows_here = T.rows - (local - lane);
          if (rows_here >= 32) {
            const int32_t y = T.row0 + local - lane;
            if constexpr (KIND == kGlu) {
              stage_limbs<LIMBS>(&maps.out[0], stage_at, lane, c0, y, f[0]);
            } else {
              stage_limbs<LIMBS>(&maps.out[0], stage_at, lane, c0, y, f[0], turn);
              stage_limbs<LIMBS>(&maps.out[1], stage_at, lane, c0, y, f[1], turn);
              stage_limbs<LIMBS>(&maps.out[2], stage_at, lane, c0, y, f[kTensors - 1], turn);
            }
          } else if (lane < rows_here) {
            // the ragged end of a subgraph: a box would reach into the next one's rows
            const int64_t at = (int64_t)(T.row0 + local) * A.out_ld + c0;
            const int width = (int)(A.out_ld - c0);
            store_limbs<LIMBS>(A.out[0] + at, A.out_limb, width, f[0]);
            if (KIND == kGluBack) {
              store_limbs<LIMBS>(A.out[1] + at, A.out_limb, width, f[1]);
              store_limbs<LIMBS>(A.out[2] + at, A.out_limb, width, f[kTensors - 1]);
            }
          }
        } else {
          // a row per lane: out[row][c0 ..], or, transposed, out[c0 + e][row]
          const bool part_sum = kAlongRows && T.slot >= 0;
          const bool wide = kAlongRows ? (part_sum || A.out_f32) : A.y_f32;
          const bool valid = kAlongRows ? T.m0 + local < A.p[T.problem].M : local < T.rows;
          const float scale = kAlongRows ? A.p[T.problem].scale : A.scale;
          const int64_t row = (kAlongRows ? T.m0 : T.row0) + local;
          if (!(KIND == kDown && A.masked)) {
#pragma unroll
            for (int e = 0; e < 32; ++e) f[0][e] *= scale;
          } else {
            const uint64_t q0 = (uint64_t)row * ((A.cols + 3) / 4) + (c0 >> 2);
#pragma unroll
            for (int q = 0; q < 8; ++q) {
              const uint4 w = words.quad(A.mask, q0 + q);
              f[0][4 * q] = w.x > A.mask.lim ? f[0][4 * q] * A.mask.scale : 0.0f;
              f[0][4 * q + 1] = w.y > A.mask.lim ? f[0][4 * q + 1] * A.mask.scale : 0.0f;
              f[0][4 * q + 2] = w.z > A.mask.lim ? f[0][4 * q + 2] * A.mask.scale : 0.0f;
              f[0][4 * q + 3] = w.w > A.mask.lim ? f[0][4 * q + 3] * A.mask.scale : 0.0f;
            }
          }
          void* out;
          int64_t ld;
          bool vectors;
          if (kAlongRows) {
            const Problem& P = A.p[T.problem];
            out = part_sum ? (void*)(A.scratch + (int64_t)T.slot * A.slot_stride + P.scratch_at)
                           : wide ? (void*)(static_cast<float*>(P.out) + T.set * P.set_stride)
                                  : (void*)(static_cast<__nv_bfloat16*>(P.out) + T.set * P.set_stride);
            ld = P.transposed ? P.M : P.N;
            vectors = (part_sum || A.out_vectors) && ld % (wide ? 4 : 8) == 0;
            if (P.transposed) {
              if (valid) {
                if (wide) {
                  float* o = static_cast<float*>(out) + (int64_t)c0 * ld + row;
#pragma unroll
                  for (int e = 0; e < 32; ++e)
                    if (c0 + e < cols) o[(int64_t)e * ld] = f[0][e];
                } else {
                  __nv_bfloat16* o = static_cast<__nv_bfloat16*>(out) + (int64_t)c0 * ld + row;
#pragma unroll
                  for (int e = 0; e < 32; ++e)
                    if (c0 + e < cols) o[(int64_t)e * ld] = __float2bfloat16_rn(f[0][e]);
                }
              }
              continue;
            }
          } else {
            out = A.y;
            ld = A.y_ld;
            vectors = A.y_vectors;
          }
          if constexpr (!kAlongRows) {
            if (vectors && T.rows - (local - lane) >= 32) {
              if constexpr (LIMBS == 1) stage_limbs<1>(&maps.out[0], stage_at, lane, c0, (int32_t)(row - lane), f[0]);
              else stage_floats(&maps.out[0], stage_at, lane, c0, (int32_t)(row - lane), f[0]);
              continue;
            }
          }
          if (vectors && c0 + 32 <= cols) {
            if (valid) {
              if (wide) {
                uint4* o = reinterpret_cast<uint4*>(static_cast<float*>(out) + row * ld + c0);
#pragma unroll
                for (int e = 0; e < 8; ++e)
                  o[e] = make_uint4(__float_as_uint(f[0][4 * e]), __float_as_uint(f[0][4 * e + 1]), __float_as_uint(f[0][4 * e + 2]),
                                    __float_as_uint(f[0][4 * e + 3]));
              } else {
                uint4* o = reinterpret_cast<uint4*>(static_cast<__nv_bfloat16*>(out) + row * ld + c0);
#pragma unroll
                for (int e = 0; e < 4; ++e)
                  o[e] = make_uint4(vio::pack_bf16(f[0][8 * e], f[0][8 * e + 1]), vio::pack_bf16(f[0][8 * e + 2], f[0][8 * e + 3]),
                                    vio::pack_bf16(f[0][8 * e + 4], f[0][8 * e + 5]), vio::pack_bf16(f[0][8 * e + 6], f[0][8 * e + 7]));
              }
            }
          } else {
            const int rows_here = (kAlongRows ? A.p[T.problem].M - T.m0 : T.rows) - (local - lane);
            if (wide) store_rows<true>(stage, lane, rows_here, row - lane, c0, cols, out, ld, f[0]);
            else store_rows<false>(stage, lane, rows_here, row - lane, c0, cols, out, ld, f[0]);
          }
        }
      }
    }
    if (!kAlongRows && lane == 0) store_box_done();
  }
  // ------------------------------------------------------------------------------------ the end
  if (*abort_flag) {
    if (threadIdx.x == 0) atomicMin(A.status, (int32_t)GNNCO_INTERNAL);
    const long long t0 = clock64();                        // copies and products already issued end before the memory goes
    while (clock64() - t0 < 1000000ll) {}
  }
  tc::tc_fence_before_sync();
  __syncthreads();
  if (PAIR) tc::cluster_sync_all();
  if (warp == 0) {
    if (PAIR) tc::tmem_dealloc_pair(tmem, 512);
    else tc::tmem_dealloc(tmem, 512);
  }
}

// -------------------------------------------------------------------------------------------- launch
template <typename Kernel>
int32_t launch_clusters(Kernel kernel, int threads, uint32_t smem, const Maps& maps, const Args& args, int clusters, int ctas, cudaStream_t st) {
  cudaLaunchConfig_t cfg{};
  cfg.gridDim = dim3(clusters * ctas);
  cfg.blockDim = dim3(threads);
  cfg.dynamicSmemBytes = smem;
  cfg.stream = st;
  cudaLaunchAttribute attr[2];
  cfg.attrs = attr;
  cfg.numAttrs = 0;
  if (args.chained) {                                      // it sets itself up while the launch before it ends
    attr[cfg.numAttrs].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[cfg.numAttrs++].val.programmaticStreamSerializationAllowed = 1;
  }
  if (ctas > 1) {
    attr[cfg.numAttrs].id = cudaLaunchAttributeClusterDimension;
    attr[cfg.numAttrs].val.clusterDim.x = ctas; attr[cfg.numAttrs].val.clusterDim.y = 1; attr[cfg.numAttrs++].val.clusterDim.z = 1;
  }
  GNNCO_CUDA_TRY(cudaLaunchKernelEx(&cfg, kernel, maps, args));
  return GNNCO_OK;
}

template <int KIND, int LIMBS, bool PAIR>
int32_t launch_one(const Maps& maps, const Args& args, int device, int sms, cudaStream_t st) {
  auto kernel = tiles<KIND, LIMBS, PAIR>;
  static std::atomic<int> allowed{0};
  const int32_t rc = allow_shared_memory(kernel, kSmem, device, allowed);
  if (rc != GNNCO_OK) return rc;
  const int most = PAIR ? resident_pairs(device, sms) : sms;
  return launch_clusters(kernel, kThreads, kSmem, maps, args, args.tiles < most ? args.tiles : most, PAIR ? 2 : 1, st);
}

}  // namespace ff
