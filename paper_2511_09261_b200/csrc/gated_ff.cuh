// Declarations shared by the translation units of the gated feed-forward block:
//
//   g = x Wg_s,  u = x Wu_s,  h = act(g) .* u,  y = drop(h Wd_s)             for the rows of every subgraph s
//
// and its gradients, with dy' the masked gradient:  dh = dy' Wd_s^T,  dg = dh .* u .* act'(g),  du = dh .* act(g),
//   dx = dg Wg_s^T + du Wu_s^T,   dWg_s = x^T dg,  dWu_s = x^T du,  dWd_s = h^T dy'      (sums over the rows of s).
// gated_ff.cu holds the entry points, the choice of kernels and the copies of operands; gated_ff_tiles.cuh the tiled products.
#pragma once

#include <cuda.h>

#include "internal.cuh"
#include "mask.cuh"

namespace ff {

// The tiled products.
//   kGlu      h                                A = x            B = Wg, Wu
//   kGluBack  h, dg, du                        A = dy', x       B = Wd (2), Wg, Wu (0, 1)
//   kDown     y                                A = h            B = Wd
//   kDx       dx                               A = dg, du       B = Wg, Wu
//   kWeights  dWg, dWu, dWd                    both operands are read along the rows that are summed
enum Kind { kGlu, kGluBack, kDown, kDx, kWeights };

struct Maps {
  CUtensorMap a[3], b[3];
  CUtensorMap out[3];                  // results in boxes of 32 rows: h, dg, du in 32 columns (16 where there are three), y or dx
                                       // in 64 bytes of columns
};

// one weight gradient: [M x N] or, transposed, [N x M] in memory
struct Problem {
  void* out;
  int64_t set_stride;                  // elements between the sets of out
  int64_t scratch_at;                  // where this gradient starts inside a slot of partial sums
  int32_t M, N, m_tiles, n_tiles, nt;
  int32_t transposed;
  float scale;
};

struct Args {
  // tiles of rows: from the handle's tables, or every TM rows (tile_row0 == nullptr)
  const int32_t *tile_row0, *tile_rows, *node_part;
  int64_t rows;
  int32_t m_tiles, n_tiles, tiles;
  int32_t nt;                          // columns of a tile (of each of g, u, dh; of y or dx)
  int32_t K[2];                        // lengths of the contractions: K[0], then K[1] (0: one only)
  int32_t cols;                        // columns of the result
  int32_t act;
  float scale;                         // of dh, y
  // results of kGlu, kGluBack: bfloat16 limbs, rows ld elements apart
  __nv_bfloat16* out[3];
  int64_t out_ld, out_limb;
  // results of kDown, kDx
  void* y;
  int64_t y_ld;
  int32_t y_f32, y_vectors;            // y_vectors: rows start and end on 16 bytes
  int32_t masked;
  philox::Mask mask;
  // kWeights
  Problem p[3];
  const int32_t *chunk_begin, *chunk_end, *chunk_slot;     // nullptr: `chunks` runs of chunk_rows rows of one set
  int32_t chunks, chunk_rows;
  int32_t per_chunk;                   // tiles of all three gradients
  int32_t out_f32, out_vectors;
  float* scratch;
  int64_t slot_stride;
  int32_t* status;
  int32_t chained;                     // a launch of the same call comes before
};

// clusters of two CTAs that the device holds at once (0: none)
int resident_pairs(int device, int sms);

}  // namespace ff

// A tensor map of bfloat16 or float32 boxes, swizzled over the bytes of a box's row where these are 128 (the layout of the MMA operands) or
// 64, plain where they are 32 (tc_gemm2.cu).
bool encode_boxes(CUtensorMap* m, bool f32, const void* base, int rank, const uint64_t* dims, const uint64_t* strides, const uint32_t* box);
