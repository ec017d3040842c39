// The gated feed-forward block, forward and backward: entry points, work areas, copies of operands and the choice of kernels
// (formulas and kinds of products: gated_ff.cuh; the products: gated_ff_tiles.cuh).
//
// Up to four rows with one set of weights: gated_ff_rows.cu.  Subgraphs of few rows in float32: gated_ff_sets.cu.  Bfloat16 forward with
// widths up to 256: gated_ff_fused.cu; backward, up to dx, with widths up to 128: gated_ff_fused_back.cu.  Else
// Forward:   [operands as limbs]   h = act(x Wg) .* (x Wu)   y = drop(h Wd)
// Backward:  [operands as limbs]   h, dg, du (g and u are computed again: nothing but x is kept from the forward pass, which at
//            widths up to some 400 is also faster than writing and reading them)   dx   the weight gradients   [their partial sums]
//
// Operands of the products are bfloat16 with rows that start on 16 bytes.  A tensor that is not (float32 features or weights, odd
// widths, unaligned views, a gradient that passes a mask first) is copied into the work area once, as one or three limbs.
// Each rounding: h, dg and du are stored as the operands of the next product, in bfloat16 features one bfloat16 (2^-8 of the value at
// most, as much as the results are rounded by), in float32 features three limbs (24 bits); float32 weights of bfloat16
// features are rounded to bfloat16.  All sums are float32, and none depends on timing.
#include "gated_ff.cuh"
#include "gated_ff_sets.cuh"
#include "vec_io.cuh"

namespace ff {
int32_t launch_tiles_bf16(Kind kind, bool pair, const Maps& maps, const Args& args, int device, int sms, cudaStream_t st);
int32_t launch_tiles_f32(Kind kind, bool pair, const Maps& maps, const Args& args, int device, int sms, cudaStream_t st);
int32_t launch_fused(const Maps& maps, const Args& args, int device, int sms, cudaStream_t st);
int32_t launch_fused_back(const Maps& maps, const CUtensorMap& dx_map, const Args& args, int device, int sms, cudaStream_t st);
bool few_rows(const gnnco_gated_ff_desc* d, int sms);
int32_t launch_few_rows(gnnco_handle* h, const gnnco_gated_ff_desc* d, const philox::Mask* mask, float* hidden, void* y, int64_t y_ld,
                        cudaStream_t st);
}  // namespace ff

namespace {

using ff::Args;
using ff::Kind;
using ff::Maps;

constexpr int kMaxWidth = 65536;

// ------------------------------------------------------------------------------ copies of operands
struct PackJob {
  const void* from;
  __nv_bfloat16* to;
  int64_t rows, from_ld, to_ld, to_limb;
  int32_t cols, from_f32, vectors, masked;
  int32_t flat;                                            // vectors, and both sides are one run of elements
};
struct PackJobs {
  PackJob j[5];
  philox::Mask mask;
};

// [rows x cols] -> LIMBS bfloat16 matrices with rows of to_ld elements (a multiple of 8; zeros behind cols): 8 columns a thread.
// A masked job keeps elements or sets them to zero and leaves the scale to the products' results, so that nothing is rounded here
// that was not before.
template <int LIMBS>
__global__ void __launch_bounds__(256) pack_operands(const __grid_constant__ PackJobs P) {
  asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
  const PackJob& J = P.j[blockIdx.y];
  const int64_t chunks = J.to_ld / 8, items = J.rows * chunks;
  philox::Stream words(P.mask);
  for (int64_t base = (int64_t)blockIdx.x * 256; base < items; base += (int64_t)gridDim.x * 256) {
    int64_t row = 0, from, to_at;
    int c = 0;
    if (J.flat) {
      from = to_at = (base + threadIdx.x) * 8;
      if (base + threadIdx.x >= items) break;
    } else {
      const int64_t row0 = base / chunks;
      const uint32_t off = (uint32_t)(base - row0 * chunks) + threadIdx.x, r = off / (uint32_t)chunks;
      row = row0 + r;
      c = (int)(off - r * (uint32_t)chunks) * 8;
      if (row >= J.rows) break;
      from = row * J.from_ld + c;
      to_at = row * J.to_ld + c;
    }
    float f[8];
    if (J.flat || (J.vectors && c + 8 <= J.cols)) {
      if (J.from_f32) {
        vio::Raw<float, 8> v;
        v.template load<true>(static_cast<const float*>(J.from) + from);
#pragma unroll
        for (int e = 0; e < 8; ++e) f[e] = v.get(e);
      } else {
        vio::Raw<__nv_bfloat16, 8> v;
        v.template load<true>(static_cast<const __nv_bfloat16*>(J.from) + from);
#pragma unroll
        for (int e = 0; e < 8; ++e) f[e] = v.get(e);
      }
    } else {
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        f[e] = 0.0f;
        if (c + e < J.cols) {
          if (J.from_f32) f[e] = static_cast<const float*>(J.from)[from + e];
          else f[e] = __bfloat162float(static_cast<const __nv_bfloat16*>(J.from)[from + e]);
        }
      }
    }
    if (J.masked) {
      uint4 two[2];
      if (J.flat) {                                        // (cols is a multiple of 8)
        words.quads(P.mask, (uint64_t)(base + threadIdx.x) * 2, two);
      } else {
        const uint64_t q = (uint64_t)row * ((J.cols + 3) / 4) + c / 4;
        two[0] = words.quad(P.mask, q);
        two[1] = words.quad(P.mask, q + 1);
      }
#pragma unroll
      for (int k = 0; k < 2; ++k) {
        const uint4 w = two[k];
        f[4 * k] = w.x > P.mask.lim ? f[4 * k] : 0.0f;
        f[4 * k + 1] = w.y > P.mask.lim ? f[4 * k + 1] : 0.0f;
        f[4 * k + 2] = w.z > P.mask.lim ? f[4 * k + 2] : 0.0f;
        f[4 * k + 3] = w.w > P.mask.lim ? f[4 * k + 3] : 0.0f;
      }
    }
    __nv_bfloat16* const to = J.to + to_at;
#pragma unroll
    for (int l = 0; l < LIMBS; ++l) {
      uint32_t w[4];
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        w[e] = vio::pack_bf16(f[2 * e], f[2 * e + 1]);
        if (l + 1 < LIMBS) {
          f[2 * e] -= vio::bf_lo(w[e]);                    // exact
          f[2 * e + 1] -= vio::bf_hi(w[e]);
        }
      }
      *reinterpret_cast<uint4*>(to + l * J.to_limb) = make_uint4(w[0], w[1], w[2], w[3]);
    }
  }
}

// ------------------------------------------------------------------- partial sums of weight gradients
struct JoinArgs {
  const float* scratch;
  int64_t slot_stride, at[3], count[3];
  void* out[3];
  const int32_t *part, *first, *slots;                     // nullptr: set 0, slots 0 .. all - 1
  int32_t all, out_f32;
};
// grid: (blocks of elements, set, gradient); the slots of a set are added in order
__global__ void __launch_bounds__(256) join_sums(const JoinArgs A) {
  const int q = blockIdx.z, k = blockIdx.y;
  const int set = A.part ? A.part[k] : 0, first = A.part ? A.first[k] : 0, slots = A.part ? A.slots[k] : A.all;
  for (int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x; i < A.count[q]; i += (int64_t)gridDim.x * 256) {
    float s = 0.0f;
    for (int j = 0; j < slots; ++j) s += A.scratch[(int64_t)(first + j) * A.slot_stride + A.at[q] + i];
    const int64_t to = (int64_t)set * A.count[q] + i;
    if (A.out_f32) static_cast<float*>(A.out[q])[to] = s;
    else static_cast<__nv_bfloat16*>(A.out[q])[to] = __float2bfloat16_rn(s);
  }
}

// ------------------------------------------------------------------------------------ tensor maps
// [limbs][rows][cols] with rows ld elements apart: boxes of `box_rows` x 64, all limbs
bool map_rows(CUtensorMap* m, const void* base, int64_t rows, int cols, int64_t ld, int64_t limb, int limbs, int box_rows) {
  const uint64_t dims[3] = {(uint64_t)cols, (uint64_t)rows, (uint64_t)limbs};
  const uint64_t strides[2] = {(uint64_t)ld * 2, (uint64_t)(limbs > 1 ? limb : ld) * 2};
  const uint32_t box[3] = {64u, (uint32_t)box_rows, (uint32_t)limbs};
  return encode_boxes(m, false, base, 3, dims, strides, box);
}
// results: boxes of 32 rows
bool map_out(CUtensorMap* m, bool f32, const void* base, int64_t rows, int cols, int64_t ld, int64_t limb, int limbs, int box_cols) {
  const uint64_t es = f32 ? 4 : 2;
  const uint64_t dims[3] = {(uint64_t)cols, (uint64_t)rows, (uint64_t)limbs};
  const uint64_t strides[2] = {(uint64_t)ld * es, (uint64_t)(limbs > 1 ? limb : ld) * es};
  const uint32_t box[3] = {(uint32_t)box_cols, 32u, 1u};
  return encode_boxes(m, f32, base, 3, dims, strides, box);
}
// [limbs][sets][rows][cols]
bool map_sets(CUtensorMap* m, const void* base, int64_t sets, int rows, int cols, int64_t ld, int limbs, int box_rows) {
  const uint64_t dims[4] = {(uint64_t)cols, (uint64_t)rows, (uint64_t)sets, (uint64_t)limbs};
  const uint64_t strides[3] = {(uint64_t)ld * 2, (uint64_t)rows * ld * 2, (uint64_t)sets * rows * ld * 2};
  const uint32_t box[4] = {64u, (uint32_t)box_rows, 1u, (uint32_t)limbs};
  return encode_boxes(m, false, base, 4, dims, strides, box);
}

// ------------------------------------------------------------------------------------ the plan of a call
struct Operand {                                           // as the products read it
  const __nv_bfloat16* p = nullptr;
  int64_t ld = 0, limb = 0;
};
int64_t up8(int64_t x) { return (x + 7) / 8 * 8; }
int64_t up16(int64_t x) { return (x + 15) / 16 * 16; }

struct Work {
  size_t x = 0, dy = 0, wg = 0, wu = 0, wd = 0, h = 0, dg = 0, du = 0, scratch = 0, total = 0;
};
constexpr size_t kNone = ~(size_t)0;

bool direct(const void* p, int64_t ld, int dtype) { return dtype == GNNCO_BF16 && ((uintptr_t)p & 15) == 0 && ld % 8 == 0; }
int limbs_of(const gnnco_gated_ff_desc* d) { return d->feat_dtype == GNNCO_F32 ? 3 : 1; }

// chunks of rows whose weight gradients are summed apart
struct Chunks {
  int32_t count = 1, rows = 0, slots = 0;
  bool table = false;
};

int64_t blocks_of(int64_t a, int64_t b) { return (a + b - 1) / b; }

// Tiles of the weight gradients.  Each gradient is summed as [M x N] or, transposed, [N x M], whichever pads less.
void shape_problem(ff::Problem* P, int32_t R, int32_t C, bool pair, bool vectors) {
  const int tm = pair ? 256 : 128;
  auto nt_of = [&](int n) { return pair ? (n > 128 ? 256 : 128) : (n > 64 ? 128 : 64); };
  auto area = [&](int m, int n) { return blocks_of(m, tm) * tm * blocks_of(n, nt_of(n)) * nt_of(n); };
  const int64_t plain = area(R, C), turned = area(C, R);
  // (as transposed, lanes hold neighbouring elements of a row whatever its alignment)
  P->transposed = turned < plain || (turned == plain && !vectors);
  P->M = P->transposed ? C : R;
  P->N = P->transposed ? R : C;
  P->nt = nt_of(P->N);
  P->m_tiles = (int32_t)blocks_of(P->M, tm);
  P->n_tiles = (int32_t)blocks_of(P->N, P->nt);
}
int64_t tiles_of(const ff::Problem* p) {
  int64_t t = 0;
  for (int q = 0; q < 3; ++q) t += (int64_t)p[q].m_tiles * p[q].n_tiles;
  return t;
}

// elements of a slot of partial sums, and where the gradients start in it
int64_t slot_layout(const gnnco_gated_ff_desc* d, int64_t at[3]) {
  const int64_t a = (int64_t)d->F * d->H, b = (int64_t)d->H * d->F_out;
  at[0] = 0;
  at[1] = (a + 63) / 64 * 64;
  at[2] = 2 * at[1];
  return at[2] + (b + 63) / 64 * 64;
}

Chunks chunks_of(const gnnco_handle* h, const gnnco_gated_ff_desc* d) {
  Chunks c;
  if (d->sets > 1) {                                       // the handle's runs of rows, at most kMostRunRows long: long subgraphs are cut
    c.table = true;
    c.count = h->all_rows.n_wg_chunks;
    c.slots = h->all_rows.n_wg_slots;
    return c;
  }
  // one set: enough runs that every SM has a tile of 128 x 128, none shorter than 512 rows and none longer than kMostRunRows
  ff::Problem p[3];
  shape_problem(p, d->F, d->H, false, true);
  p[1] = p[0];
  shape_problem(p + 2, d->H, d->F_out, false, true);
  const int64_t tiles = tiles_of(p);
  int64_t runs = tiles >= h->sm_count ? 1 : blocks_of(h->sm_count, tiles);
  if (runs > blocks_of(d->rows, 512)) runs = blocks_of(d->rows, 512);
  if (runs < blocks_of(d->rows, kMostRunRows)) runs = blocks_of(d->rows, kMostRunRows);
  if (runs < 1) runs = 1;
  c.rows = (int32_t)((blocks_of(d->rows, runs) + 63) / 64 * 64);
  c.count = c.rows > 0 ? (int32_t)blocks_of(d->rows, c.rows) : 1;
  c.slots = c.count > 1 ? c.count : 0;
  return c;
}

// Both products in one kernel (gated_ff_fused.cu) or in two?  One pair of CTAs walks all of H there, so it takes tiles of 256 rows for half of
// the pairs, or a short H.  (Device time with cold caches, one kernel and two: 12,000 x 256 x 512 18.0 and 21.1 us, x 4,096 76 and
// 86; 1,000 x 64 x 128 in 8 sets 9.0 and 13.1; but 4,000 x 256 x 512 16.3 and 14.3, 4,000 x 256 x 4,096 71 and 38.)
bool fuses(const gnnco_handle* h, const gnnco_gated_ff_desc* d) {
  if (d->feat_dtype != GNNCO_BF16 || d->F > 256 || d->F_out > 256) return false;
  const int64_t pairs = ff::resident_pairs(h->device, h->sm_count), tiles = d->sets > 1 ? h->all_rows.n_pairs : blocks_of(d->rows, 256);
  return pairs > 0 && (2 * tiles >= pairs || d->H <= 256);
}

// The same for h, dg, du and dx (gated_ff_fused_back.cu): where H is short, since a chunk of H costs more there (its weights are read for 128
// rows, by pairs of CTAs for 256).  Backward passes, in one kernel and in two, in us: 1.13 M x 128 x 256 in 1,024 sets 1,220 and 1,320,
// 300,000 x 32 x 64 in 512 113 and 125, 1,000 x 64 x 128 in 8 20.5 and 22.6, 4,000 x 128 x 256 32.7 and 32.8; but 60,000 x 64 x 600 in
// 64 170 and 166, 20,000 x 128 x 1,024 133 and 117, and with few tiles 300 x 128 x 256 24.6 and 22.6.
// dx is written there before the weight gradients read x and dy, so it must be neither of them; without weight gradients it may lie over
// them row by row (a tile's rows are read before they are written, other tiles' rows at any time).
bool fuses_back(const gnnco_handle* h, const gnnco_gated_ff_desc* d, const gnnco_gated_ff_grads* g, const Operand& x, const Operand& dy) {
  if (d->feat_dtype != GNNCO_BF16 || d->F > 128 || d->F_out > 128 || d->H > 256 || !g->dx || ((uintptr_t)g->dx & 15) || g->dx_ld % 8 || d->F % 8)
    return false;
  auto apart = [&](const Operand& o, int cols) {
    const uintptr_t a = (uintptr_t)g->dx, b = (uintptr_t)o.p;
    return a + ((d->rows - 1) * g->dx_ld + d->F) * 2 <= b || b + ((d->rows - 1) * o.ld + cols) * 2 <= a;
  };
  // row r of dx touches no row of o but r
  auto by_rows = [&](const Operand& o, int cols) {
    const int64_t off = (int64_t)((uintptr_t)g->dx - (uintptr_t)o.p), ld = g->dx_ld;
    return d->rows == 1 || (o.ld == ld && off <= (ld - d->F) * 2 && off >= (cols - ld) * 2);
  };
  auto fits = [&](const Operand& o, int cols) { return apart(o, cols) || (!g->dw_gate && by_rows(o, cols)); };
  if (!fits(x, d->F) || !fits(dy, d->F_out)) return false;
  const int64_t tiles = d->sets > 1 ? h->all_rows.n_tiles : blocks_of(d->rows, 128);
  return 4 * tiles >= h->sm_count || d->H <= 128;
}

Work lay_out(const gnnco_handle* h, const gnnco_gated_ff_desc* d, bool backward) {
  Work w;
  const int64_t limbs = limbs_of(d), sets = d->sets;
  if (!backward && ff::few_rows(d, h->sm_count)) {         // h in float32
    w.h = 0;
    w.total = align_up((size_t)d->rows * d->H * 4);
    return w;
  }
  if (!backward && ff::few_rows_per_set(h, d)) {           // (backward the weight gradients' type decides, which is not known here)
    w.h = 0;
    w.total = align_up((size_t)d->rows * d->H * 4);
    return w;
  }
  auto take = [&](bool needed, int64_t elements) {
    if (!needed) return kNone;
    const size_t at = w.total;
    w.total += align_up((size_t)elements * 2);
    return at;
  };
  w.x = take(!direct(d->x, d->x_ld, d->feat_dtype), limbs * d->rows * up8(d->F));
  w.wg = take(!direct(d->w_gate, d->H, d->w_dtype), limbs * sets * d->F * up8(d->H));
  w.wu = take(!direct(d->w_up, d->H, d->w_dtype), limbs * sets * d->F * up8(d->H));
  w.wd = take(!direct(d->w_down, d->F_out, d->w_dtype), limbs * sets * d->H * up8(d->F_out));
  w.h = take(backward || !fuses(h, d), limbs * d->rows * up16(d->H));
  if (backward) {
    w.dg = take(true, limbs * d->rows * up16(d->H));
    w.du = take(true, limbs * d->rows * up16(d->H));
    w.dy = take(true, limbs * d->rows * up8(d->F_out));    // (whether dy itself will do is not known here)
    int64_t at[3];
    w.scratch = take(true, 2 * (int64_t)chunks_of(h, d).slots * slot_layout(d, at));
  }
  if (w.total < 256) w.total = 256;
  return w;
}

int32_t check(const gnnco_handle* h, const gnnco_gated_ff_desc* d, philox::Mask* mask, bool* drops) {
  if (!h || !d || d->rows < 0 || d->F < 1 || d->H < 1 || d->F_out < 1) return GNNCO_INVALID_ARGUMENT;
  if (d->feat_dtype != GNNCO_F32 && d->feat_dtype != GNNCO_BF16) return GNNCO_UNSUPPORTED;
  if (d->w_dtype != GNNCO_F32 && (d->w_dtype != GNNCO_BF16 || d->feat_dtype != GNNCO_BF16)) return GNNCO_UNSUPPORTED;
  if (d->F > kMaxWidth || d->H > kMaxWidth || d->F_out > kMaxWidth || d->rows > 0x7fffff00ll) return GNNCO_UNSUPPORTED;
  if (d->act != GNNCO_SILU && d->act != GNNCO_GELU && d->act != GNNCO_RELU) return GNNCO_INVALID_ARGUMENT;
  if (d->sets != 1 && (d->sets != h->S || d->rows != h->n)) return GNNCO_INVALID_ARGUMENT;
  if (mask && d->drop && !make_mask(d->drop, mask, drops)) return GNNCO_INVALID_ARGUMENT;
  return GNNCO_OK;
}

struct Call {
  gnnco_handle* h;
  const gnnco_gated_ff_desc* d;
  cudaStream_t st;
  int limbs;
  bool drops;                                              // whether the mask drops anything
  bool launched;                                           // by this call, so far
  PackJobs jobs;
  int n_jobs = 0;

  ff::SetArgs set_args() const {
    ff::SetArgs A = {};
    A.x = static_cast<const float*>(d->x);
    A.x_ld = d->x_ld;
    A.wg = static_cast<const float*>(d->w_gate);
    A.wu = static_cast<const float*>(d->w_up);
    A.wd = static_cast<const float*>(d->w_down);
    A.F = d->F; A.H = d->H; A.F_out = d->F_out;
    A.act = d->act;
    A.masked = drops;
    A.mask = jobs.mask;
    return A;
  }
  Operand operand(const void* p, int64_t rows, int32_t cols, int64_t ld, int dtype, bool masked, char* copy) {
    Operand o;
    if (!masked && direct(p, ld, dtype)) {
      o.p = static_cast<const __nv_bfloat16*>(p);
      o.ld = ld;
      return o;
    }
    o.p = reinterpret_cast<__nv_bfloat16*>(copy);
    o.ld = up8(cols);
    o.limb = rows * o.ld;
    PackJob& j = jobs.j[n_jobs++];
    j.from = p;
    j.to = reinterpret_cast<__nv_bfloat16*>(copy);
    j.rows = rows; j.from_ld = ld; j.to_ld = o.ld; j.to_limb = o.limb;
    j.cols = cols; j.from_f32 = dtype == GNNCO_F32; j.masked = masked;
    j.vectors = ((uintptr_t)p & 15) == 0 && ld % (dtype == GNNCO_F32 ? 4 : 8) == 0;
    j.flat = j.vectors && ld == cols && cols % 8 == 0;
    return o;
  }
  void pack() {
    if (n_jobs == 0) return;
    int64_t most = 0;
    for (int k = 0; k < n_jobs; ++k) {
      const int64_t b = blocks_of(jobs.j[k].rows * (jobs.j[k].to_ld / 8), 256);
      if (b > most) most = b;
    }
    const int64_t cap = (int64_t)h->sm_count * 16;
    const dim3 grid((unsigned)(most < cap ? most : cap), n_jobs);
    if (limbs == 3) pack_operands<3><<<grid, 256, 0, st>>>(jobs);
    else pack_operands<1><<<grid, 256, 0, st>>>(jobs);
    h->launches += 1;
    launched = true;
  }
  // tiles of rows
  int64_t row_tiles(bool pair) const {
    if (d->sets > 1) return pair ? h->all_rows.n_pairs : h->all_rows.n_tiles;
    return blocks_of(d->rows, pair ? 256 : 128);
  }
  void rows_of(Args* a, bool pair) const {
    a->rows = d->rows;
    a->node_part = h->node_part;
    a->m_tiles = (int32_t)row_tiles(pair);
    if (d->sets > 1) {
      a->tile_row0 = pair ? h->all_rows.pair_row0 : h->all_rows.tile_row0;
      a->tile_rows = pair ? h->all_rows.pair_rows : h->all_rows.tile_rows;
    }
    a->status = h->status;
  }
  int32_t launch(Kind kind, bool pair, const Maps& maps, Args* a, int64_t tiles) {
    if (tiles > 0x7ff00000) return GNNCO_UNSUPPORTED;      // (a tile's number plus two rounds of the grid stays in 32 bits)
    a->tiles = (int32_t)tiles;
    a->chained = launched;
    launched = true;
    const int32_t rc = limbs == 3 ? ff::launch_tiles_f32(kind, pair, maps, *a, h->device, h->sm_count, st)
                                  : ff::launch_tiles_bf16(kind, pair, maps, *a, h->device, h->sm_count, st);
    if (rc == GNNCO_OK) h->launches += 1;
    return rc;
  }
  // Pairs of CTAs halve what is read per product; single CTAs with tiles of a quarter of the size spread small calls over more SMs and
  // leave less of the last round idle.  Rounds of tiles times their length, in cycles: the products of a stage (64 of the contraction)
  // or its copies at the 45 bytes a cycle that an SM got from L2, and some 2,500 at the ends that nothing covers.
  // (Backward by pairs and by singles: 1.13 M x 128 x 256 bfloat16 1,330 and 1,419 us, 4,039 x 128 x 343 float32 in 16 sets 82 and 68.)
  bool use_pairs(int64_t pair_tiles, int64_t single_tiles, int64_t stages, int pair_cols, int single_cols) const {
    const int64_t pairs = ff::resident_pairs(h->device, h->sm_count), sms = h->sm_count;
    if (pairs <= 0 || pair_tiles < pairs) return false;
    const int64_t products = limbs == 3 ? 6 : 1;
    auto stage = [&](int cols, int staged) {
      const int64_t multiply = products * cols * 2, copy = (int64_t)limbs * (128 + staged) * 128 / 45;
      return multiply > copy ? multiply : copy;
    };
    const int64_t by_pairs = blocks_of(pair_tiles, pairs) * (stages * stage(pair_cols, pair_cols / 2) + 2500);
    const int64_t by_singles = blocks_of(single_tiles, sms) * (stages * stage(single_cols, single_cols) + 2500);
    return by_pairs <= by_singles;
  }

  // h (and, with dy, dg and du) from x
  int32_t gates(const Operand& x, const Operand* dy, const Operand& wg, const Operand& wu, const Operand& wd, const Operand* out) {
    auto nt_of = [&](bool pair) { return pair && (dy ? limbs == 1 : d->H > 64) ? 128 : 64; };
    // (columns that are multiplied per stage: g and u, on average two of g, u and dh)
    const bool pair = use_pairs(row_tiles(true) * blocks_of(d->H, nt_of(true)), row_tiles(false) * blocks_of(d->H, nt_of(false)),
                                blocks_of(d->F, 64) + (dy ? blocks_of(d->F_out, 64) : 0), dy ? nt_of(true) * 3 / 2 : nt_of(true) * 2,
                                dy ? nt_of(false) * 3 / 2 : nt_of(false) * 2);
    Args a = {};
    Maps m = {};
    rows_of(&a, pair);
    a.nt = nt_of(pair);
    a.n_tiles = (int32_t)blocks_of(d->H, a.nt);
    a.K[0] = dy ? d->F_out : d->F;
    a.K[1] = dy ? d->F : 0;
    a.cols = d->H;
    a.act = d->act;
    a.scale = dy && drops ? jobs.mask.scale : 1.0f;
    for (int k = 0; k < (dy ? 3 : 1); ++k) a.out[k] = const_cast<__nv_bfloat16*>(out[k].p);
    a.out_ld = out[0].ld;
    a.out_limb = out[0].limb;
    bool ok = map_rows(&m.a[dy ? 1 : 0], x.p, d->rows, d->F, x.ld, x.limb, limbs, 128) &&
              map_sets(&m.b[0], wg.p, d->sets, d->F, d->H, wg.ld, limbs, 64) && map_sets(&m.b[1], wu.p, d->sets, d->F, d->H, wu.ld, limbs, 64);
    if (dy)
      ok = ok && map_rows(&m.a[0], dy->p, d->rows, d->F_out, dy->ld, dy->limb, limbs, 128) &&
           map_sets(&m.b[2], wd.p, d->sets, d->H, d->F_out, wd.ld, limbs, pair ? a.nt / 2 : a.nt);
    for (int k = 0; k < (dy ? 3 : 1); ++k)
      ok = ok && map_out(&m.out[k], false, out[k].p, d->rows, d->H, out[k].ld, out[k].limb, limbs, dy ? 16 : 32);
    if (!ok) return GNNCO_CUDA_ERROR;
    return launch(dy ? ff::kGluBack : ff::kGlu, pair, m, &a, (int64_t)a.m_tiles * a.n_tiles);
  }
  bool wide_pairs(int cols, int64_t stages) const {
    const int p = wide_tile(true, cols), q = wide_tile(false, cols);
    return use_pairs(row_tiles(true) * blocks_of(cols, p), row_tiles(false) * blocks_of(cols, q), stages, p, q);
  }
  // columns of a tile of y or dx: wide, but for single CTAs that would leave half of the GPU idle (dx of 4,039 x 128 in 16 subgraphs: 32
  // tiles of 128 columns or 64 of 64, the whole backward pass 71.5 or 68.2 us; 3,000 x 512: 96 or 192 tiles, 77.2 or 83.5 us)
  int wide_tile(bool pair, int cols) const {
    if (pair) return cols > 128 ? 256 : 128;
    return cols > 64 && 2 * row_tiles(false) * blocks_of(cols, 128) > h->sm_count ? 128 : 64;
  }

  // y = drop(h Wd)
  int32_t down(const Operand& hh, const Operand& wd, void* y, int64_t y_ld) {
    const bool pair = wide_pairs(d->F_out, blocks_of(d->H, 64));
    Args a = {};
    Maps m = {};
    rows_of(&a, pair);
    a.nt = wide_tile(pair, d->F_out);
    a.n_tiles = (int32_t)blocks_of(d->F_out, a.nt);
    a.K[0] = d->H;
    if (!result(&a, &m, y, y_ld, d->F_out)) return GNNCO_CUDA_ERROR;
    a.masked = drops;
    a.mask = jobs.mask;
    if (!map_rows(&m.a[0], hh.p, d->rows, d->H, hh.ld, hh.limb, limbs, 128) ||
        !map_sets(&m.b[0], wd.p, d->sets, d->H, d->F_out, wd.ld, limbs, 64))
      return GNNCO_CUDA_ERROR;
    return launch(ff::kDown, pair, m, &a, (int64_t)a.m_tiles * a.n_tiles);
  }
  int32_t fused(const Operand& x, const Operand& wg, const Operand& wu, const Operand& wd, void* y, int64_t y_ld) {
    Args a = {};
    Maps m = {};
    rows_of(&a, true);
    a.n_tiles = 1;
    a.K[0] = d->F;
    a.K[1] = d->H;
    a.act = d->act;
    if (!result(&a, &m, y, y_ld, d->F_out)) return GNNCO_CUDA_ERROR;
    a.masked = drops;
    a.mask = jobs.mask;
    a.tiles = a.m_tiles;
    a.chained = launched;
    if (!map_rows(&m.a[0], x.p, d->rows, d->F, x.ld, x.limb, 1, 128) || !map_sets(&m.b[0], wg.p, d->sets, d->F, d->H, wg.ld, 1, 64) ||
        !map_sets(&m.b[1], wu.p, d->sets, d->F, d->H, wu.ld, 1, 64) || !map_sets(&m.b[2], wd.p, d->sets, d->H, d->F_out, wd.ld, 1, 64))
      return GNNCO_CUDA_ERROR;
    const int32_t rc = ff::launch_fused(m, a, h->device, h->sm_count, st);
    if (rc == GNNCO_OK) h->launches += 1;
    return rc;
  }
  // h, dg, du (where they are wanted) and dx
  int32_t gates_and_dx(const Operand& x, const Operand& dy, const Operand& wg, const Operand& wu, const Operand& wd, const Operand* out,
                       bool keep, void* dx, int64_t dx_ld) {
    Args a = {};
    Maps m = {};
    CUtensorMap dx_map;
    rows_of(&a, false);
    a.n_tiles = 1;
    a.K[0] = d->F_out;
    a.K[1] = d->H;
    a.cols = d->F;
    a.act = d->act;
    a.scale = drops ? jobs.mask.scale : 1.0f;
    a.y = dx;
    a.y_ld = dx_ld;
    a.out_ld = out[0].ld;
    a.tiles = a.m_tiles;
    a.chained = launched;
    launched = true;
    bool ok = map_rows(&m.a[0], x.p, d->rows, d->F, x.ld, 0, 1, 128) && map_rows(&m.a[1], dy.p, d->rows, d->F_out, dy.ld, 0, 1, 128) &&
              map_sets(&m.b[0], wg.p, d->sets, d->F, d->H, wg.ld, 1, d->F > 64 ? 128 : 64) &&
              map_sets(&m.b[1], wu.p, d->sets, d->F, d->H, wu.ld, 1, d->F > 64 ? 128 : 64) &&
              map_sets(&m.b[2], wd.p, d->sets, d->H, d->F_out, wd.ld, 1, 64) && map_out(&dx_map, false, dx, d->rows, d->F, dx_ld, 0, 1, 16);
    for (int k = 0; keep && k < 3; ++k) {
      a.out[k] = const_cast<__nv_bfloat16*>(out[k].p);
      ok = ok && map_out(&m.out[k], false, out[k].p, d->rows, d->H, out[k].ld, 0, 1, 64);
    }
    if (!ok) return GNNCO_CUDA_ERROR;
    const int32_t rc = ff::launch_fused_back(m, dx_map, a, h->device, h->sm_count, st);
    if (rc == GNNCO_OK) h->launches += 1;
    return rc;
  }
  // dx = dg Wg^T + du Wu^T
  int32_t input_grad(const Operand& dg, const Operand& du, const Operand& wg, const Operand& wu, void* dx, int64_t dx_ld) {
    const bool pair = wide_pairs(d->F, 2 * blocks_of(d->H, 64));
    Args a = {};
    Maps m = {};
    rows_of(&a, pair);
    a.nt = wide_tile(pair, d->F);
    a.n_tiles = (int32_t)blocks_of(d->F, a.nt);
    a.K[0] = a.K[1] = d->H;
    if (!result(&a, &m, dx, dx_ld, d->F)) return GNNCO_CUDA_ERROR;
    const int box = pair ? a.nt / 2 : a.nt;
    if (!map_rows(&m.a[0], dg.p, d->rows, d->H, dg.ld, dg.limb, limbs, 128) || !map_rows(&m.a[1], du.p, d->rows, d->H, du.ld, du.limb, limbs, 128) ||
        !map_sets(&m.b[0], wg.p, d->sets, d->F, d->H, wg.ld, limbs, box) || !map_sets(&m.b[1], wu.p, d->sets, d->F, d->H, wu.ld, limbs, box))
      return GNNCO_CUDA_ERROR;
    return launch(ff::kDx, pair, m, &a, (int64_t)a.m_tiles * a.n_tiles);
  }
  bool result(Args* a, Maps* m, void* y, int64_t ld, int32_t cols) const {
    a->cols = cols;
    a->scale = 1.0f;
    a->y = y;
    a->y_ld = ld;
    a->y_f32 = d->feat_dtype == GNNCO_F32;
    // (a box is cut at the tensor's last column in units of 16 bytes: rows that end inside one would lose what lies behind them)
    a->y_vectors = ((uintptr_t)y & 15) == 0 && ld % (a->y_f32 ? 4 : 8) == 0 && cols % (a->y_f32 ? 4 : 8) == 0;
    return !a->y_vectors || map_out(&m->out[0], a->y_f32, y, d->rows, cols, ld, 0, 1, a->y_f32 ? 16 : 32);
  }
  int32_t weight_grads(const Operand& x, const Operand& dy, const Operand* hdd, const gnnco_gated_ff_grads* g, float* scratch) {
    const Chunks c = chunks_of(h, d);
    const bool f32 = g->dw_dtype == GNNCO_F32;
    void* const outs[3] = {g->dw_gate, g->dw_up, g->dw_down};
    const int32_t R[3] = {d->F, d->F, d->H}, C[3] = {d->H, d->H, d->F_out};
    const Operand row_op[3] = {x, x, hdd[0]}, col_op[3] = {hdd[1], hdd[2], dy};
    Args a = {};
    Maps m = {};
    rows_of(&a, false);
    a.tile_row0 = nullptr;
    a.out_f32 = f32;
    a.out_vectors = 1;
    for (int q = 0; q < 3; ++q)
      if (((uintptr_t)outs[q] & 15) || (int64_t)R[q] * C[q] % 8) a.out_vectors = 0;
    auto shape = [&](bool pair) {
      for (int q = 0; q < 3; ++q) shape_problem(&a.p[q], R[q], C[q], pair, a.out_vectors && C[q] % 8 == 0);
      return (int64_t)c.count * tiles_of(a.p);
    };
    const int64_t rows_of_chunk = blocks_of(d->rows, c.count > 0 ? c.count : 1);
    const int64_t pair_tiles = shape(true), single_tiles = shape(false);
    const bool pair = use_pairs(pair_tiles, single_tiles, blocks_of(rows_of_chunk, 64), 256, 128);
    const int64_t tiles = shape(pair);
    int64_t at[3];
    a.slot_stride = slot_layout(d, at);
    a.scratch = scratch;
    a.chunks = c.count;
    a.chunk_rows = c.rows;
    a.per_chunk = (int32_t)tiles_of(a.p);
    if (c.table) {
      a.chunk_begin = h->all_rows.wg_begin;
      a.chunk_end = h->all_rows.wg_end;
      a.chunk_slot = h->all_rows.wg_slot;
    }
    for (int q = 0; q < 3; ++q) {
      ff::Problem& P = a.p[q];
      P.out = outs[q];
      P.set_stride = (int64_t)R[q] * C[q];
      P.scratch_at = at[q];
      P.scale = q == 2 && drops ? jobs.mask.scale : 1.0f;
      const Operand& A = P.transposed ? col_op[q] : row_op[q];
      const Operand& B = P.transposed ? row_op[q] : col_op[q];
      if (!map_rows(&m.a[q], A.p, d->rows, P.M, A.ld, A.limb, limbs, 64) || !map_rows(&m.b[q], B.p, d->rows, P.N, B.ld, B.limb, limbs, 64))
        return GNNCO_CUDA_ERROR;
    }
    const int32_t rc = launch(ff::kWeights, pair, m, &a, tiles);
    if (rc != GNNCO_OK) return rc;
    if (c.slots > 0) {
      JoinArgs J = {};
      J.scratch = scratch;
      J.slot_stride = a.slot_stride;
      int64_t most = 0;
      for (int q = 0; q < 3; ++q) {
        J.at[q] = at[q];
        J.count[q] = (int64_t)R[q] * C[q];
        J.out[q] = outs[q];
        if (J.count[q] > most) most = J.count[q];
      }
      if (c.table) { J.part = h->all_rows.wg_mpart; J.first = h->all_rows.wg_mfirst; J.slots = h->all_rows.wg_mcount; }
      J.all = c.slots;
      J.out_f32 = f32;
      const int sets = c.table ? h->all_rows.n_wg_multi : 1;
      const int64_t blocks = blocks_of(most, 256);
      // (a split subgraph has over 2,048 rows: there are fewer than 2^20 of them, and a grid takes 65,535 at a time)
      for (int s0 = 0; s0 < sets; s0 += 65535) {
        JoinArgs K = J;
        if (c.table) { K.part += s0; K.first += s0; K.slots += s0; }
        join_sums<<<dim3((unsigned)(blocks < 1024 ? blocks : 1024), sets - s0 < 65535 ? sets - s0 : 65535, 3), 256, 0, st>>>(K);
        h->launches += 1;
      }
    }
    return GNNCO_OK;
  }
};

}  // namespace

extern "C" int32_t gnnco_gated_ff_workspace_bytes(const gnnco_handle* h, const gnnco_gated_ff_desc* d, int32_t backward, size_t* bytes) {
  if (!bytes) return GNNCO_INVALID_ARGUMENT;
  const int32_t rc = check(h, d, nullptr, nullptr);
  if (rc != GNNCO_OK) return rc;
  *bytes = lay_out(h, d, backward != 0).total;
  return GNNCO_OK;
}

extern "C" int32_t gnnco_gated_ff(gnnco_handle* h, const gnnco_gated_ff_desc* d, void* y, int64_t y_ld, void* ws, size_t ws_bytes,
                                  void* stream) {
  Call c = {};
  const int32_t rc = check(h, d, &c.jobs.mask, &c.drops);
  if (rc != GNNCO_OK) return rc;
  if (d->rows == 0) return GNNCO_OK;
  if (!d->x || d->x_ld < d->F || !d->w_gate || !d->w_up || !d->w_down || !y || y_ld < d->F_out || !ws || ((uintptr_t)ws & 255) ||
      !on_own_device(h))
    return GNNCO_INVALID_ARGUMENT;
  // (a row of y would lie over other rows of x, which one of the kernels reads while it writes y)
  if (y == d->x && y_ld != d->x_ld && d->rows > 1) return GNNCO_INVALID_ARGUMENT;
  const Work w = lay_out(h, d, false);
  if (ws_bytes < w.total) return GNNCO_WORKSPACE_TOO_SMALL;
  c.h = h;
  c.d = d;
  c.st = static_cast<cudaStream_t>(stream);
  c.limbs = limbs_of(d);
  ProfScope prof_(h, K_GATED_FF, c.st);
  char* const base = static_cast<char*>(ws);
  if (ff::few_rows(d, h->sm_count)) {
    const int32_t r = ff::launch_few_rows(h, d, c.drops ? &c.jobs.mask : nullptr, reinterpret_cast<float*>(base + w.h), y, y_ld, c.st);
    if (r != GNNCO_OK) return r;
    GNNCO_LAUNCH_CHECK();
    return GNNCO_OK;
  }
  const int64_t sets = d->sets;
  if (ff::few_rows_per_set(h, d)) {
    ff::SetArgs A = c.set_args();
    A.h = reinterpret_cast<float*>(base + w.h);
    A.out = static_cast<float*>(y);
    A.out_ld = y_ld;
    const int32_t r = ff::launch_sets(h, A, sets, false, c.st);
    if (r != GNNCO_OK) return r;
    GNNCO_LAUNCH_CHECK();
    return GNNCO_OK;
  }
  const Operand x = c.operand(d->x, d->rows, d->F, d->x_ld, d->feat_dtype, false, base + w.x);
  const Operand wg = c.operand(d->w_gate, sets * d->F, d->H, d->H, d->w_dtype, false, base + w.wg);
  const Operand wu = c.operand(d->w_up, sets * d->F, d->H, d->H, d->w_dtype, false, base + w.wu);
  const Operand wd = c.operand(d->w_down, sets * d->H, d->F_out, d->F_out, d->w_dtype, false, base + w.wd);
  Operand hh;
  hh.p = reinterpret_cast<__nv_bfloat16*>(base + w.h);
  hh.ld = up16(d->H);
  hh.limb = d->rows * hh.ld;
  c.pack();
  int32_t r;
  if (fuses(h, d)) {
    r = c.fused(x, wg, wu, wd, y, y_ld);
  } else {
    r = c.gates(x, nullptr, wg, wu, wd, &hh);
    if (r == GNNCO_OK) r = c.down(hh, wd, y, y_ld);
  }
  if (r != GNNCO_OK) return r;
  GNNCO_LAUNCH_CHECK();
  return GNNCO_OK;
}

extern "C" int32_t gnnco_gated_ff_backward(gnnco_handle* h, const gnnco_gated_ff_desc* d, const void* dy, int64_t dy_ld,
                                           const gnnco_gated_ff_grads* g, void* ws, size_t ws_bytes, void* stream) {
  Call c = {};
  const int32_t rc = check(h, d, &c.jobs.mask, &c.drops);
  if (rc != GNNCO_OK) return rc;
  const bool weights = g && g->dw_gate;
  if (!g || weights != (g->dw_up != nullptr) || weights != (g->dw_down != nullptr)) return GNNCO_INVALID_ARGUMENT;
  if (weights && g->dw_dtype != GNNCO_F32 && g->dw_dtype != GNNCO_BF16) return GNNCO_UNSUPPORTED;
  if (!on_own_device(h)) return GNNCO_INVALID_ARGUMENT;
  c.h = h;
  c.d = d;
  c.st = static_cast<cudaStream_t>(stream);
  c.limbs = limbs_of(d);
  const int64_t sets = d->sets;
  if (d->rows == 0) {                                      // sums of nothing (rows are never 0 with a set per subgraph)
    if (!weights) return GNNCO_OK;
    const size_t es = g->dw_dtype == GNNCO_F32 ? 4 : 2;
    GNNCO_CUDA_TRY(cudaMemsetAsync(g->dw_gate, 0, (size_t)d->F * d->H * es, c.st));
    GNNCO_CUDA_TRY(cudaMemsetAsync(g->dw_up, 0, (size_t)d->F * d->H * es, c.st));
    GNNCO_CUDA_TRY(cudaMemsetAsync(g->dw_down, 0, (size_t)d->H * d->F_out * es, c.st));
    return GNNCO_OK;
  }
  if (!d->x || d->x_ld < d->F || !d->w_gate || !d->w_up || !d->w_down || !dy || dy_ld < d->F_out || (g->dx && g->dx_ld < d->F) ||
      (!g->dx && !weights) || !ws || ((uintptr_t)ws & 255))
    return GNNCO_INVALID_ARGUMENT;
  const Work w = lay_out(h, d, true);
  if (ws_bytes < w.total) return GNNCO_WORKSPACE_TOO_SMALL;
  ProfScope prof_(h, K_GATED_FF, c.st);
  char* const base = static_cast<char*>(ws);
  if (ff::few_rows_per_set(h, d) && (!weights || g->dw_dtype == GNNCO_F32)) {
    ff::SetArgs A = c.set_args();
    A.dy = static_cast<const float*>(dy);
    A.dy_ld = dy_ld;
    if (g->dx) {                                           // (the tiled products' copies of h, dg and du take more)
      A.dg = reinterpret_cast<float*>(base + w.h);
      A.du = A.dg + d->rows * d->H;
    }
    A.dwg = static_cast<float*>(g->dw_gate);
    A.dwu = static_cast<float*>(g->dw_up);
    A.dwd = static_cast<float*>(g->dw_down);
    A.out = static_cast<float*>(g->dx);
    A.out_ld = g->dx_ld;
    const int32_t r = ff::launch_sets(h, A, sets, true, c.st);
    if (r != GNNCO_OK) return r;
    GNNCO_LAUNCH_CHECK();
    return GNNCO_OK;
  }
  const Operand x = c.operand(d->x, d->rows, d->F, d->x_ld, d->feat_dtype, false, base + w.x);
  const Operand wg = c.operand(d->w_gate, sets * d->F, d->H, d->H, d->w_dtype, false, base + w.wg);
  const Operand wu = c.operand(d->w_up, sets * d->F, d->H, d->H, d->w_dtype, false, base + w.wu);
  const Operand wd = c.operand(d->w_down, sets * d->H, d->F_out, d->F_out, d->w_dtype, false, base + w.wd);
  const Operand dyo = c.operand(dy, d->rows, d->F_out, dy_ld, d->feat_dtype, c.drops, base + w.dy);
  Operand hdd[3];
  const size_t at[3] = {w.h, w.dg, w.du};
  for (int k = 0; k < 3; ++k) {
    hdd[k].p = reinterpret_cast<__nv_bfloat16*>(base + at[k]);
    hdd[k].ld = up16(d->H);
    hdd[k].limb = d->rows * hdd[k].ld;
  }
  c.pack();
  const bool fused = fuses_back(h, d, g, x, dyo);
  int32_t r = fused ? c.gates_and_dx(x, dyo, wg, wu, wd, hdd, weights, g->dx, g->dx_ld) : c.gates(x, &dyo, wg, wu, wd, hdd);
  if (r == GNNCO_OK && weights) r = c.weight_grads(x, dyo, hdd, g, reinterpret_cast<float*>(base + w.scratch));
  // (last: dx may be x or dy)
  if (r == GNNCO_OK && g->dx && !fused) r = c.input_grad(hdd[1], hdd[2], wg, wu, g->dx, g->dx_ld);
  if (r != GNNCO_OK) return r;
  GNNCO_LAUNCH_CHECK();
  return GNNCO_OK;
}
