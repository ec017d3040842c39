// Input embeddings shared between nodes: every node carries a token (a degree class, a community, a type) and reads row
// token[i] of one table.
//
//   gnnco_embedding_lookup   out[i] = scale * T[token[i]]
//   gnnco_embedding_plan     stable order of the rows by token (built once per token vector)
//   gnnco_embedding_grad     dT[v] = scale * sum_{i: token[i] = v} dout[i]
//
// Both passes are bound by memory: the lookup writes rows * F elements and reads the table through L2, the gradient
// reads rows * F elements once and writes V * F.  The gradient uses no floating-point atomics: rows are visited in token
// order, which fixes the order of every sum (bit-identical from run to run) and keeps the running sum of a token in
// registers however often the token occurs.
#include <atomic>

#include "internal.cuh"
#include "vec_io.cuh"

namespace {

// -------------------------------------------------------------------------------------------------------- lookup

// A warp owns a tile of `tile` rows whose tokens it reads in one coalesced load; eight loads are in flight per lane.  Calls with
// few rows use 4-row tiles to spread over the SMs.  Two forms:
//   lookup_rows    rows of 2^i (up to 32) or a multiple of 32 vectors: `width` lanes per row, so a lane's column never changes
//   lookup_kernel  any other width: the lanes walk the tile's vectors as one flat list
// (10M x 256 bf16: 904 us, 983 in the flat form, whose index arithmetic takes two thirds of the issue slots.)
template <typename TT, typename TO, int VEC>
__global__ void __launch_bounds__(256) lookup_rows(const int32_t* __restrict__ tokens, const TT* __restrict__ table, int64_t table_ld,
                                                   TO* __restrict__ out, int64_t out_ld, int64_t rows, int32_t V,
                                                   int32_t vecs_per_row, int32_t width, float scale, int tile, int32_t* status) {
  const int lane = threadIdx.x & 31;
  const int64_t row0 = ((int64_t)blockIdx.x * 8 + (threadIdx.x >> 5)) * tile;
  if (row0 >= rows) return;
  const int here = (int)min((int64_t)tile, rows - row0);
  int32_t tok = lane < here ? __ldcs(tokens + row0 + lane) : -1;
  if (tok >= V) {
    atomicMin(status, (int32_t)GNNCO_OUT_OF_RANGE);
    tok = -1;
  }
  const int step = 32 / width, sub = lane / width;          // rows per load of the warp, this lane's of them
  constexpr int U = 8;
  for (int j = lane % width; j < vecs_per_row; j += width) {
    const TT* const src = table + (int64_t)j * VEC;
    TO* dst = out + (row0 + sub) * out_ld + (int64_t)j * VEC;
    const int64_t hop = step * out_ld;
    for (int r = sub; r < here + sub; r += U * step) {      // (the same number of rounds for all lanes)
      vio::Raw<TT, VEC> v[U];
#pragma unroll
      for (int k = 0; k < U; ++k) {
        const int32_t t = __shfl_sync(0xffffffffu, tok, (r + k * step) & 31);
        if (r + k * step < here && t >= 0) v[k].template load<false>(src + t * table_ld);
        else v[k].zero();
      }
#pragma unroll
      for (int k = 0; k < U; ++k) {
        if (r + k * step < here) vio::store_stream<TO, VEC>(dst, vio::mul(vio::Vec<VEC>(v[k]), scale).v);
        dst += hop;
      }
    }
  }
}

template <typename TT, typename TO, int VEC>
__global__ void __launch_bounds__(256) lookup_kernel(const int32_t* __restrict__ tokens, const TT* __restrict__ table,
                                                     int64_t table_ld, TO* __restrict__ out, int64_t out_ld, int64_t rows,
                                                     int32_t V, int32_t vecs_per_row, float scale, int tile,
                                                     int32_t* status) {
  const int lane = threadIdx.x & 31;
  const int64_t row0 = ((int64_t)blockIdx.x * 8 + (threadIdx.x >> 5)) * tile;
  if (row0 >= rows) return;
  const int here = (int)min((int64_t)tile, rows - row0);
  int32_t tok = lane < here ? __ldcs(tokens + row0 + lane) : -1;
  if (tok >= V) {
    atomicMin(status, (int32_t)GNNCO_OUT_OF_RANGE);
    tok = -1;
  }
  const uint32_t vpr = (uint32_t)vecs_per_row, total = (uint32_t)here * vpr;
  // (row, vector) of this lane's next element, stepped by 32 without dividing again
  const uint32_t dr = 32 / vpr, dj = 32 % vpr;
  uint32_t rn = lane / vpr, jn = lane % vpr;
  constexpr int U = 8;
  for (uint32_t base = 0; base < total; base += 32 * U) {
    vio::Raw<TT, VEC> v[U];
    uint32_t r[U], j[U];
#pragma unroll
    for (int k = 0; k < U; ++k) {
      const uint32_t q = base + 32 * k + lane;
      r[k] = rn;
      j[k] = jn;
      rn += dr;
      jn += dj;
      if (jn >= vpr) { jn -= vpr; ++rn; }
      const int32_t t = __shfl_sync(0xffffffffu, tok, (int)(r[k] & 31));
      if (q < total && t >= 0) v[k].template load<false>(table + (int64_t)t * table_ld + (int64_t)j[k] * VEC);
      else v[k].zero();
    }
#pragma unroll
    for (int k = 0; k < U; ++k) {
      if (base + 32 * k + lane >= total) continue;
      vio::store_stream<TO, VEC>(out + (row0 + r[k]) * out_ld + (int64_t)j[k] * VEC, vio::mul(vio::Vec<VEC>(v[k]), scale).v);
    }
  }
}

template <typename TT, typename TO, int VEC>
void lookup_vec(const int32_t* tokens, const TT* table, int64_t table_ld, TO* out, int64_t out_ld, int64_t rows, int32_t V, int32_t F,
                float scale, int tile, unsigned grid, int32_t* status, cudaStream_t st) {
  const int vecs = F / VEC;
  if (vecs % 32 == 0 || 32 % vecs == 0)
    lookup_rows<TT, TO, VEC><<<grid, 256, 0, st>>>(tokens, table, table_ld, out, out_ld, rows, V, vecs, vecs < 32 ? vecs : 32, scale, tile, status);
  else
    lookup_kernel<TT, TO, VEC><<<grid, 256, 0, st>>>(tokens, table, table_ld, out, out_ld, rows, V, vecs, scale, tile, status);
}

template <typename TT, typename TO>
int32_t lookup_typed(gnnco_handle* h, const int32_t* tokens, const TT* table, int64_t table_ld, TO* out, int64_t out_ld,
                     int64_t rows, int32_t V, int32_t F, float scale, cudaStream_t st) {
  const int tile = rows >= (int64_t)h->sm_count * 256 ? 32 : 4;
  const unsigned grid = (unsigned)((rows + 8 * tile - 1) / (8 * tile));
  auto fits = [&](int vec) {
    return F % vec == 0 && vec_ok(table, table_ld, sizeof(TT), vec) && vec_ok(out, out_ld, sizeof(TO), vec);
  };
  if (fits(8) && (sizeof(TT) == 2 || sizeof(TO) == 2))
    lookup_vec<TT, TO, 8>(tokens, table, table_ld, out, out_ld, rows, V, F, scale, tile, grid, h->status, st);
  else if (fits(4))
    lookup_vec<TT, TO, 4>(tokens, table, table_ld, out, out_ld, rows, V, F, scale, tile, grid, h->status, st);
  else if (fits(2))
    lookup_vec<TT, TO, 2>(tokens, table, table_ld, out, out_ld, rows, V, F, scale, tile, grid, h->status, st);
  else
    lookup_vec<TT, TO, 1>(tokens, table, table_ld, out, out_ld, rows, V, F, scale, tile, grid, h->status, st);
  h->launches += 1;
  GNNCO_LAUNCH_CHECK();
  return GNNCO_OK;
}

// ---------------------------------------------------------------------------------------------------- order by token
//
// Stable least-significant-digit radix sort of the row numbers by token, at most 10 bits per pass and only as many bits as
// V has, shared evenly over the passes (17 bits: 9 + 8): two passes up to a million tokens.
// A fixed number of blocks owns one contiguous span of positions each: block histograms (digit-major), one block per
// digit scans that digit's row, and the scatter puts a tile in digit order in shared memory before it writes it out, so
// that a digit's rows leave together.  Rows without a token get key V and end up last.
constexpr int kOrdThreads = 512, kOrdWarps = kOrdThreads / 32, kOrdRounds = 8;
constexpr int kOrdTile = kOrdThreads * kOrdRounds;         // positions of one block-wide step
constexpr int kOrdMaxBlocks = 444;                         // 3 per SM: all resident at once
// Up to here no separate scan: every block adds up the block counts itself, which saves a launch per pass and costs reads that grow with
// the blocks (with and without the scan: one pass of 10 bits 12.2 and 10.8 us over 4 blocks, 13.5 and 14.7 over 12, 14.0 and 24.5 over 25;
// two passes 22.4 and 19.2, 22.7 and 20.2, 22.9 and 24.0).
constexpr int kOrdFewBlocks = 12;
constexpr int kOrdMaxBits = 10, kOrdMaxDigits = 1 << kOrdMaxBits;
constexpr int kSmallRows = 4096;                           // up to here one block sorts everything in shared memory

struct PlanLayout {
  int32_t *key_a, *idx_a, *key_b, *idx_b, *hist, *totals;
  uint32_t* present;
  int32_t* runs;                                           // small plans only: number of runs, their first positions, the last one's end
  float* partial;                                          // [chunks][2][F]
  size_t bytes;
  int64_t chunks;
  int chunk;
  int passes, bits;                                        // bits per pass
};

int bits_of(int64_t x) {                                   // bits needed for values 0 .. x
  int b = 0;
  while (((int64_t)1 << b) <= x) ++b;
  return b;
}

// Positions of one chunk of the gradient: enough chunks to fill the GPU some times over, at most 256 so that a token's
// partial sums stay few, at least 16 so that the chunk boundaries (a partial row each) do not outweigh the rows.
int chunk_of(int64_t rows) {
  int c = 16;
  while (c < 256 && rows / (2 * c) >= 148 * 64) c *= 2;
  return c;
}

// Few rows: one block sorts, and one block per token that occurs adds its rows.
bool is_small(int64_t rows) { return rows > 0 && rows <= kSmallRows; }

PlanLayout plan_layout(void* ws, int64_t rows, int32_t V, int32_t F) {
  Carver c(ws, 0);
  PlanLayout L;
  L.passes = (bits_of(V) + kOrdMaxBits - 1) / kOrdMaxBits;
  L.bits = (bits_of(V) + L.passes - 1) / L.passes;
  if (L.bits < 1) L.bits = 1;
  L.chunk = chunk_of(rows);
  L.chunks = (rows + L.chunk - 1) / L.chunk;
  L.key_a = c.take<int32_t>(rows);
  L.idx_a = c.take<int32_t>(rows);
  L.key_b = c.take<int32_t>(rows);
  L.idx_b = c.take<int32_t>(rows);
  L.hist = c.take<int32_t>(kOrdMaxDigits * (size_t)kOrdMaxBlocks);
  L.totals = c.take<int32_t>(kOrdMaxDigits);
  L.present = c.take<uint32_t>(((size_t)V + 31) / 32);
  L.runs = c.take<int32_t>(is_small(rows) ? rows + 2 : 0);
  L.partial = c.take<float>((size_t)L.chunks * 2 * F);
  L.bytes = c.off;
  return L;
}
// the buffers that hold the result after `passes` passes
const int32_t* plan_keys(const PlanLayout& L) { return (L.passes & 1) ? L.key_a : L.key_b; }
const int32_t* plan_rows(const PlanLayout& L) { return (L.passes & 1) ? L.idx_a : L.idx_b; }

__device__ __forceinline__ int32_t token_key(int32_t t, int32_t V) { return (uint32_t)t < (uint32_t)V ? t : V; }

// lanes of the warp with the same digit (one ballot per bit: match.any serialises over the distinct digits)
template <int MOST>
__device__ __forceinline__ uint32_t same_digit(uint32_t d, int bits, bool valid) {
  uint32_t peers = __ballot_sync(0xffffffffu, valid);
#pragma unroll
  for (int b = 0; b < MOST; ++b) {
    if (b >= bits) break;
    const uint32_t one = (d >> b) & 1u;
    peers &= __ballot_sync(0xffffffffu, one) ^ (one - 1u);   // lanes with the same bit as this one
  }
  return peers;
}

// FIRST: keys come from the token vector (row number = position); tokens are checked.
template <bool FIRST>
__global__ void __launch_bounds__(kOrdThreads) order_histogram(const int32_t* __restrict__ keys, int64_t N, int64_t span,
                                                               int shift, int digits, int32_t V, int32_t* __restrict__ hist,
                                                               uint32_t* present, int32_t* status) {
  __shared__ int32_t cnt[kOrdMaxDigits];
  for (int d = threadIdx.x; d < digits; d += kOrdThreads) cnt[d] = 0;
  __syncthreads();
  if (FIRST)                                               // the gradient marks the tokens that occur
    for (int64_t w = (int64_t)blockIdx.x * kOrdThreads + threadIdx.x; w < ((int64_t)V + 31) / 32; w += (int64_t)gridDim.x * kOrdThreads)
      present[w] = 0u;
  const int64_t lo = (int64_t)blockIdx.x * span, hi = min(N, lo + span);
  bool wrong = false;
  for (int64_t p0 = lo; p0 < hi; p0 += kOrdThreads * 4) {
    int32_t k[4];
#pragma unroll
    for (int u = 0; u < 4; ++u) {
      const int64_t p = p0 + u * kOrdThreads + threadIdx.x;
      k[u] = p < hi ? keys[p] : -2;
    }
#pragma unroll
    for (int u = 0; u < 4; ++u) {
      if (p0 + u * kOrdThreads + threadIdx.x >= hi) continue;
      if (FIRST) {
        wrong |= k[u] >= V;
        k[u] = token_key(k[u], V);
      }
      atomicAdd(&cnt[(k[u] >> shift) & (digits - 1)], 1);
    }
  }
  if (FIRST && wrong) atomicMin(status, (int32_t)GNNCO_OUT_OF_RANGE);
  __syncthreads();
  for (int d = threadIdx.x; d < digits; d += kOrdThreads) hist[(int64_t)d * gridDim.x + blockIdx.x] = cnt[d];
}

// One block per digit: exclusive prefix of the digit's block counts (in place) and the digit's total.
__global__ void __launch_bounds__(1024) order_scan(int32_t* hist, int32_t* totals, int nblocks) {
  __shared__ int32_t warp_tot[32];
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  const int32_t x = (int)threadIdx.x < nblocks ? hist[(int64_t)blockIdx.x * nblocks + threadIdx.x] : 0;
  int32_t incl = x;
#pragma unroll
  for (int d = 1; d < 32; d <<= 1) {
    const int32_t o = __shfl_up_sync(0xffffffffu, incl, d);
    if (lane >= d) incl += o;
  }
  if (lane == 31) warp_tot[warp] = incl;
  __syncthreads();
  int32_t off = 0, tot = 0;
  for (int w = 0; w < (int)blockDim.x / 32; ++w) {
    if (w < warp) off += warp_tot[w];
    tot += warp_tot[w];
  }
  if ((int)threadIdx.x < nblocks) hist[(int64_t)blockIdx.x * nblocks + threadIdx.x] = off + incl - x;
  if (threadIdx.x == 0) totals[blockIdx.x] = tot;
}

// exclusive prefix over the block's threads (all call it; warp_tot holds one value per warp)
__device__ __forceinline__ int32_t scan_block(int32_t x, int32_t* warp_tot) {
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  int32_t incl = x;
#pragma unroll
  for (int d = 1; d < 32; d <<= 1) {
    const int32_t o = __shfl_up_sync(0xffffffffu, incl, d);
    if (lane >= d) incl += o;
  }
  if (lane == 31) warp_tot[warp] = incl;
  __syncthreads();
  int32_t off = 0;
#pragma unroll
  for (int w = 0; w < kOrdWarps; ++w)
    if (w < warp) off += warp_tot[w];
  __syncthreads();
  return off + incl - x;
}

// Thread t owns digits 2 t and 2 t + 1.
template <bool FIRST>
__global__ void __launch_bounds__(kOrdThreads, 3) order_scatter(const int32_t* __restrict__ keys, const int32_t* __restrict__ idx,
                                                             int32_t* __restrict__ keys_out, int32_t* __restrict__ idx_out,
                                                             uint32_t N, uint32_t span, int shift, int bits, int32_t V,
                                                             const int32_t* __restrict__ hist, const int32_t* __restrict__ totals) {
  extern __shared__ int32_t sm[];
  const int digits = 1 << bits;
  const uint32_t digit_mask = (uint32_t)digits - 1u;
  int32_t* const sk = sm;                                  // the tile in digit order
  int32_t* const si = sm + kOrdTile;
  int32_t* const next = sm + 2 * kOrdTile;                 // [digits] where a digit's next row goes, less its place in the tile
  int32_t* const warp_tot = next + kOrdMaxDigits;
  uint32_t* const cnt = reinterpret_cast<uint32_t*>(warp_tot + kOrdWarps);   // [warps][digits] 16-bit counters, two to a word
  uint16_t* const cnt16 = reinterpret_cast<uint16_t*>(cnt);
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, t = threadIdx.x, words = digits / 2;
  const bool owns = t < words;
  int32_t at0, at1;                                        // of digits 2 t and 2 t + 1
  {
    // the digit's total over all blocks, and its rows in the blocks before this one
    int32_t a = 0, b = 0, a_before = 0, b_before = 0;
    if (owns) {
      const int32_t* const ha = hist + (int64_t)(2 * t) * gridDim.x;
      const int32_t* const hb = ha + gridDim.x;
      if (totals) {
        a = totals[2 * t];
        b = totals[2 * t + 1];
        a_before = ha[blockIdx.x];
        b_before = hb[blockIdx.x];
      } else {
#pragma unroll 4
        for (unsigned q = 0; q < gridDim.x; ++q) {
          const int32_t x = ha[q], y = hb[q];
          a += x;
          b += y;
          if (q < blockIdx.x) {
            a_before += x;
            b_before += y;
          }
        }
      }
    }
    at0 = scan_block(a + b, warp_tot) + a_before;
    at1 = at0 - a_before + a + b_before;
  }
  const uint32_t lo = blockIdx.x * span, hi = min(N, lo + span);   // positions stay below 2^32: N < 2^31
  for (uint32_t p0 = lo; p0 < hi; p0 += kOrdTile) {
    for (int q = t; q < kOrdWarps * words; q += kOrdThreads) cnt[q] = 0;
    __syncthreads();
    // ranks inside the warp's 256 consecutive positions, in position order
    int32_t k[kOrdRounds];
    int rank[kOrdRounds];
    const uint32_t wbase = p0 + warp * (32 * kOrdRounds) + lane;
#pragma unroll
    for (int r = 0; r < kOrdRounds; ++r) {
      const uint32_t p = wbase + r * 32;
      k[r] = p < hi ? (FIRST ? token_key(keys[p], V) : keys[p]) : 0;
    }
    uint16_t* const mine = cnt16 + warp * digits;
#pragma unroll
    for (int r = 0; r < kOrdRounds; ++r) {
      const bool valid = wbase + r * 32 < hi;
      const uint32_t d = ((uint32_t)k[r] >> shift) & digit_mask;
      const uint32_t peers = same_digit<kOrdMaxBits>(d, bits, valid);
      const int before = __popc(peers & ((1u << lane) - 1u));
      rank[r] = valid ? mine[d] + before : 0;
      __syncwarp();
      if (valid && before == 0) mine[d] += (uint16_t)__popc(peers);
      __syncwarp();
    }
    int32_t v[kOrdRounds];
#pragma unroll
    for (int r = 0; r < kOrdRounds; ++r) {
      const uint32_t p = wbase + r * 32;
      v[r] = FIRST ? (int32_t)p : (p < hi ? idx[p] : 0);
    }
    __syncthreads();
    uint32_t total = 0;                                    // both digits at once: neither passes 16 bits
    if (owns)
#pragma unroll
      for (int w = 0; w < kOrdWarps; ++w) total += cnt[w * words + t];
    const int32_t n0 = (int32_t)(total & 0xffffu), n1 = (int32_t)(total >> 16);
    const int32_t first0 = scan_block(n0 + n1, warp_tot), first1 = first0 + n0;   // the digits' places in the tile
    if (owns) {
      uint32_t c = (uint32_t)first0 | ((uint32_t)first1 << 16);
#pragma unroll
      for (int w = 0; w < kOrdWarps; ++w) {
        const uint32_t n = cnt[w * words + t];
        cnt[w * words + t] = c;
        c += n;
      }
      next[2 * t] = at0 - first0;
      next[2 * t + 1] = at1 - first1;
      at0 += n0;
      at1 += n1;
    }
    __syncthreads();
#pragma unroll
    for (int r = 0; r < kOrdRounds; ++r) {
      if (wbase + r * 32 < hi) {
        const int32_t q = mine[((uint32_t)k[r] >> shift) & digit_mask] + rank[r];
        sk[q] = k[r];
        si[q] = v[r];
      }
    }
    __syncthreads();
    const int here = (int)min((uint32_t)kOrdTile, hi - p0);
#pragma unroll
    for (int r = 0; r < kOrdRounds; ++r) {
      const int q = r * kOrdThreads + t;
      if (q < here) {
        const int32_t key = sk[q], to = next[((uint32_t)key >> shift) & digit_mask] + q;
        keys_out[to] = key;
        idx_out[to] = si[q];
      }
    }
    __syncthreads();
  }
}
constexpr size_t kScatterSmem = (size_t)(2 * kOrdTile + kOrdMaxDigits + kOrdWarps + kOrdWarps * kOrdMaxDigits / 2) * sizeof(int32_t);

// All passes in one block for up to kSmallRows rows: 32 warps x 128 positions, 5 bits per pass, so that the 32 x 32 counters
// (digit-major) are one per thread and one scan over the block places everything.
constexpr int kSmallThreads = 1024, kSmallRounds = kSmallRows / kSmallThreads;
__global__ void __launch_bounds__(kSmallThreads) order_small(const int32_t* __restrict__ tokens, int32_t N, int32_t V, int bits,
                                                             int32_t* __restrict__ keys_out, int32_t* __restrict__ idx_out,
                                                             uint32_t* present, bool clear_present, int32_t* __restrict__ runs,
                                                             int32_t* status) {
  __shared__ int32_t sk[kSmallRows], si[kSmallRows];
  __shared__ int32_t cnt[32 * 33];                         // [digit][warp]
  __shared__ int32_t tot[32];
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  int32_t k[kSmallRounds], v[kSmallRounds];
  const int wbase = warp * (32 * kSmallRounds);
  if (clear_present)
    for (int32_t w = threadIdx.x; w < (V + 31) / 32; w += kSmallThreads) present[w] = 0u;
#pragma unroll
  for (int r = 0; r < kSmallRounds; ++r) {
    const int p = wbase + r * 32 + lane;
    const int32_t t = p < N ? tokens[p] : -1;
    if (t >= V) atomicMin(status, (int32_t)GNNCO_OUT_OF_RANGE);
    k[r] = token_key(t, V);
    v[r] = p;
  }
  for (int shift = 0; shift < bits; shift += 5) {
    cnt[lane * 33 + warp] = 0;
    __syncwarp();                                          // a warp counts in its own column
    int rank[kSmallRounds];
#pragma unroll
    for (int r = 0; r < kSmallRounds; ++r) {
      const bool valid = wbase + r * 32 + lane < N;
      const uint32_t d = (uint32_t)(k[r] >> shift) & 31u;
      const uint32_t peers = same_digit<5>(d, 5, valid);
      const int before = __popc(peers & ((1u << lane) - 1u));
      rank[r] = valid ? cnt[d * 33 + warp] + before : 0;
      __syncwarp();
      if (valid && before == 0) cnt[d * 33 + warp] += __popc(peers);
      __syncwarp();
    }
    __syncthreads();
    // warp w scans digit w over the warps, then the digits' totals
    const int32_t c = cnt[warp * 33 + lane];
    int32_t incl = c;
#pragma unroll
    for (int d = 1; d < 32; d <<= 1) {
      const int32_t o = __shfl_up_sync(0xffffffffu, incl, d);
      if (lane >= d) incl += o;
    }
    if (lane == 31) tot[warp] = incl;
    __syncthreads();
    int32_t before = lane < warp ? tot[lane] : 0;
#pragma unroll
    for (int d = 16; d > 0; d >>= 1) before += __shfl_xor_sync(0xffffffffu, before, d);
    cnt[warp * 33 + lane] = before + incl - c;
    __syncthreads();
#pragma unroll
    for (int r = 0; r < kSmallRounds; ++r) {
      if (wbase + r * 32 + lane < N) {
        const int at = cnt[((k[r] >> shift) & 31) * 33 + warp] + rank[r];
        sk[at] = k[r];
        si[at] = v[r];
      }
    }
    __syncthreads();
#pragma unroll
    for (int r = 0; r < kSmallRounds; ++r) {
      const int p = wbase + r * 32 + lane;
      k[r] = p < N ? sk[p] : 0;
      v[r] = p < N ? si[p] : 0;
    }
  }
  // where runs begin, numbered in order
  uint32_t heads[kSmallRounds];
  int32_t here = 0;
#pragma unroll
  for (int r = 0; r < kSmallRounds; ++r) {
    const int p = wbase + r * 32 + lane;
    const bool head = p < N && k[r] < V && (p == 0 || sk[p - 1] != k[r]);
    if (p < N) {
      keys_out[p] = k[r];
      idx_out[p] = v[r];
    }
    if (head) atomicOr(present + (k[r] >> 5), 1u << (k[r] & 31));
    heads[r] = __ballot_sync(0xffffffffu, head);
    here += __popc(heads[r]);
  }
  __syncthreads();                                         // (tot is free again)
  if (lane == 0) tot[warp] = here;
  __syncthreads();
  int32_t all = tot[lane], at = lane < warp ? all : 0;
#pragma unroll
  for (int d = 16; d > 0; d >>= 1) {
    at += __shfl_xor_sync(0xffffffffu, at, d);
    all += __shfl_xor_sync(0xffffffffu, all, d);
  }
#pragma unroll
  for (int r = 0; r < kSmallRounds; ++r) {
    const int p = wbase + r * 32 + lane;
    if ((heads[r] >> lane) & 1u) runs[1 + at + __popc(heads[r] & ((1u << lane) - 1u))] = p;
    at += __popc(heads[r]);
    // the position after the last row with a token ends the last run
    if (p < N && k[r] < V && (p == N - 1 || sk[p + 1] >= V)) {
      runs[0] = all;
      runs[1 + all] = p + 1;
    }
  }
  if (threadIdx.x == 0 && sk[0] >= V) runs[0] = 0;
}

// ------------------------------------------------------------------------------------------------------ gradient
//
// The sorted positions are cut into chunks of equal length, one team of TEAM lanes per chunk and block of TEAM * VEC
// columns, so a token that holds a third of all rows costs no more than a thousand small ones.  A run that lies inside a
// chunk goes straight to the table; the pieces of a run that crosses a chunk boundary meet in `partial`:
// slot 0 = the chunk's first run, begun in an earlier chunk; slot 1 = its last run, begun here and continued in the next.
// A block whose chunks all lie inside one run (a token with thousands of rows) adds its teams' sums first and leaves them in
// slot 0 of its first chunk.  The second kernel also writes the zero rows of tokens that do not occur.

// One bit per token that occurs, where its run begins in the sorted keys.
constexpr int kMarkPer = 8;
__device__ __forceinline__ void mark_present(const int32_t* __restrict__ keys, int64_t N, int32_t V, int64_t block, uint32_t* present) {
  const int64_t p0 = block * (256 * kMarkPer) + threadIdx.x;
  int32_t k[kMarkPer], before[kMarkPer];
#pragma unroll
  for (int u = 0; u < kMarkPer; ++u) {
    const int64_t p = p0 + u * 256;
    k[u] = p < N ? keys[p] : V;
    before[u] = p < N && p > 0 ? keys[p - 1] : -1;
  }
#pragma unroll
  for (int u = 0; u < kMarkPer; ++u)
    if (k[u] < V && before[u] != k[u]) atomicOr(present + (k[u] >> 5), 1u << (k[u] & 31));
}

// Whether chunks [c, c + group) all exist and hold nothing but one token, whose run began before them.
__device__ __forceinline__ bool is_solid(const int32_t* __restrict__ keys, int64_t N, int32_t V, int64_t c, int group, int chunk,
                                         int64_t chunks) {
  if (c == 0 || c + group > chunks) return false;
  const int32_t k = keys[c * chunk - 1];
  return k < V && keys[min(N, (c + group) * chunk) - 1] == k;
}

// Rows in flight against blocks per SM, ordering included: 10M x 256 bf16 takes 1,441 us with eight rows at four blocks (1,456 with four
// at five), 1.13M x 128 float32 166 us with four rows at five blocks (172 with eight at four); more blocks spill registers (2,370 and
// 187 us at six).  Eight rows at three blocks take 1,389 us, but 198 instead of 144 us for 4M x 64 bf16 over 300 tokens.
// A lane holds K vectors, TEAM vectors apart (narrow vectors: more columns per visit of a row).  The blocks after the last chunk
// mark the tokens that occur.
template <typename T, typename TO, int VEC, int TEAM, int K>
__global__ void __launch_bounds__(256, K == 1 && VEC < 8 ? 5 : 4) grad_chunks(const T* __restrict__ dout, int64_t dout_ld, const int32_t* __restrict__ keys,
                                                   const int32_t* __restrict__ idx, int64_t N, int32_t V, int32_t F, float scale,
                                                   int chunk, int64_t chunks, unsigned chunk_blocks, uint32_t* present,
                                                   float* __restrict__ partial, TO* __restrict__ out, int64_t out_ld) {
  constexpr int TEAMS = 256 / TEAM, W = TEAM * VEC * K;    // columns of a block
  constexpr int U = VEC >= 8 ? 8 : 4;
  if (blockIdx.x >= chunk_blocks) {
    if (blockIdx.y == 0) mark_present(keys, N, V, blockIdx.x - chunk_blocks, present);
    return;
  }
  const int tl = threadIdx.x % TEAM, team = threadIdx.x / TEAM;
  const int col0 = blockIdx.y * W + tl * VEC;              // vector q of this lane: column col0 + q TEAM VEC
  const int64_t cb = (int64_t)blockIdx.x * TEAMS, c = cb + team;
  // one run from before this block's first position to its last (the same answer for the whole block)
  const bool solid = is_solid(keys, N, V, cb, TEAMS, chunk, chunks);
  if (c >= chunks) return;                                 // whole teams leave together (shuffles below name the team); never of a solid block
  const uint32_t mask = TEAM == 32 ? 0xffffffffu : ((1u << TEAM) - 1u) << ((threadIdx.x & 31) / TEAM * TEAM);
  const int64_t p0 = c * chunk, p1 = min(N, p0 + chunk);
  vio::Vec<VEC> acc[K];
#pragma unroll
  for (int q = 0; q < K; ++q) acc[q] = vio::Vec<VEC>(0.0f);
  int32_t cur = keys[p0];
  bool head = p0 > 0 && keys[p0 - 1] == cur;
  auto to_table = [&]() {
#pragma unroll
    for (int q = 0; q < K; ++q)
      if (col0 + q * TEAM * VEC < F)
        vio::store_stream<TO, VEC>(out + (int64_t)cur * out_ld + col0 + q * TEAM * VEC, vio::mul(acc[q], scale).v);
  };
  auto to_partial = [&](int slot) {
#pragma unroll
    for (int q = 0; q < K; ++q) {
      float* const p = partial + (c * 2 + slot) * F + col0 + q * TEAM * VEC;
#pragma unroll
      for (int e = 0; e < VEC; ++e)
        if (col0 + q * TEAM * VEC < F) p[e] = acc[q].v[e];
    }
  };
  for (int64_t pb = p0; pb < p1 && cur < V; pb += TEAM) {
    const int64_t mine = pb + tl;
    const int32_t k_l = mine < p1 ? keys[mine] : V;
    const int32_t i_l = mine < p1 ? idx[mine] : 0;
#pragma unroll 1
    for (int j0 = 0; j0 < TEAM; j0 += U) {
      vio::Raw<T, VEC> v[U][K];
      int32_t k[U];
#pragma unroll
      for (int u = 0; u < U; ++u) {
        k[u] = __shfl_sync(mask, k_l, j0 + u, TEAM);
        const int32_t i = __shfl_sync(mask, i_l, j0 + u, TEAM);
        const T* const row = dout + (int64_t)i * dout_ld + col0;
#pragma unroll
        for (int q = 0; q < K; ++q) {
          if (col0 + q * TEAM * VEC < F && k[u] < V) v[u][q].template load<true>(row + q * TEAM * VEC);
          else v[u][q].zero();
        }
      }
#pragma unroll
      for (int u = 0; u < U; ++u) {
        if (k[u] != cur) {                                 // uniform over the team
          const bool real = pb + j0 + u < p1;
          if (cur < V && real) {
            if (head) to_partial(0);
            else to_table();
          }
          if (real) {
            head = false;
            cur = k[u];
#pragma unroll
            for (int q = 0; q < K; ++q) acc[q] = vio::Vec<VEC>(0.0f);
          }
        }
#pragma unroll
        for (int q = 0; q < K; ++q)
#pragma unroll
          for (int e = 0; e < VEC; ++e) acc[q].v[e] += v[u][q].get(e);
      }
    }
  }
  if (solid) {
    __shared__ float sums[TEAMS][W];
#pragma unroll
    for (int q = 0; q < K; ++q)
#pragma unroll
      for (int e = 0; e < VEC; ++e) sums[team][(q * TEAM + tl) * VEC + e] = acc[q].v[e];
    __syncthreads();
    for (int q = threadIdx.x; q < W; q += 256) {
      const int f = blockIdx.y * W + q;
      float t = 0.0f;
#pragma unroll
      for (int k = 0; k < TEAMS; ++k) t += sums[k][q];
      if (f < F) partial[cb * 2 * F + f] = t;
    }
    return;
  }
  if (cur >= V) return;
  const bool goes_on = p1 < N && keys[p1] == cur;
  if (head) to_partial(0);
  else if (goes_on) to_partial(1);
  else to_table();
}

// Runs that cross chunk boundaries: warp w of a block looks at chunk c0 + w; where a run begins there that continues, its
// pieces are slot 1 of chunk c, slot 0 of the following chunks, and slot 0 of the first chunk of every solid group of
// `group` chunks.  Up to four pieces are added by the warp, in order; more by the whole block: `wide` threads side by side
// cover the columns, the 1,024 / wide rows of threads take every so-manieth piece, and their sums are added in order.
// The blocks after the last chunk write the zero rows, 32 tokens per warp.
constexpr int kCombineWarps = 32;
struct Pieces {                                            // the pieces after the first, in order
  int64_t c1;                                              // chunks c1 .. q0 - 1, then the groups from q0 on, then chunks
  int32_t lead, groups, tail;
  int group;
  __device__ __forceinline__ int32_t count() const { return lead + groups + tail; }
  __device__ __forceinline__ int64_t chunk(int32_t i) const {
    if (i < lead) return c1 + i;
    const int32_t g = i - lead;
    return g < groups ? c1 + lead + (int64_t)g * group : c1 + lead + (int64_t)groups * group + (g - groups);
  }
};
template <typename TO>
__global__ void __launch_bounds__(kCombineWarps * 32) grad_combine(const int32_t* __restrict__ keys, int64_t N, int32_t V, int32_t F,
                                                                   float scale, int chunk, int64_t chunks, int group, int wide,
                                                                   bool vec4, unsigned chunk_blocks,
                                                                   const uint32_t* __restrict__ present,
                                                                   const float* __restrict__ partial, TO* __restrict__ out,
                                                                   int64_t out_ld) {
  __shared__ Pieces run[kCombineWarps];                    // the runs that the whole block adds, in any order: [big_runs]
  __shared__ int64_t run_chunk[kCombineWarps];
  __shared__ int32_t run_key[kCombineWarps], big_runs;
  __shared__ float sums[kCombineWarps * 32];
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  if (blockIdx.x >= chunk_blocks) {
    const int64_t v0 = ((int64_t)(blockIdx.x - chunk_blocks) * kCombineWarps + warp) * 32;
    if (v0 >= V) return;
    uint32_t gone = ~present[v0 >> 5];
    if (V - v0 < 32) gone &= (1u << (V - v0)) - 1u;
    const float z[4] = {0.0f, 0.0f, 0.0f, 0.0f};
    while (gone) {
      const int b = __ffs(gone) - 1;
      gone &= gone - 1;
      TO* const row = out + (v0 + b) * out_ld;
      if (vec4) {
        for (int col = 4 * lane; col < F; col += 128) vio::store_stream<TO, 4>(row + col, z);
      } else {
        const float z1[1] = {0.0f};
        for (int col = lane; col < F; col += 32) vio::store_stream<TO, 1>(row + col, z1);
      }
    }
    return;
  }
  if (threadIdx.x == 0) big_runs = 0;
  __syncthreads();
  const int64_t c0 = (int64_t)blockIdx.x * kCombineWarps, c = c0 + warp;
  Pieces r = {c + 1, 0, 0, 0, group};
  int32_t key = V;
  if (c < chunks) {
    // everything that decides the common case is asked for at once
    const int64_t p0 = c * chunk, p1 = min(N, p0 + chunk), p2 = min(N, p1 + chunk);
    const int32_t k_first = keys[p0], k_before = p0 > 0 ? keys[p0 - 1] : -1, k_after = p1 < N ? keys[p1] : -1;
    const int32_t k_third = p2 < N ? keys[p2] : -1;
    key = keys[p1 - 1];
    if (key < V && k_after == key && !(k_first == key && k_before == key)) {
      // how many of the following chunks begin with the key: 32 probes at a time into a sorted list
      int64_t at = c + 1, left = chunks - at;
      if (k_third != key) {
        at += 1;
        left = 0;
      }
      while (left > 0) {
        const int64_t stride = (left + 31) / 32, probe = at + lane * stride;
        const bool same = lane * stride < left && keys[probe * chunk] == key;
        const int hits = __popc(__ballot_sync(0xffffffffu, same));
        if (hits == 0) break;
        const int64_t past = (hits - 1) * stride + 1;      // this many are known to match; the next miss is within a stride
        at += past;
        left = min(stride - 1, left - past);
      }
      // [c + 1, at) begin with the key; all but perhaps the last hold nothing else
      const int64_t full = keys[min(N, at * chunk) - 1] == key ? at : at - 1;
      const int64_t q0 = (c + group) & ~(int64_t)(group - 1);   // group is a power of two
      const int64_t groups = full > q0 ? (full - q0) >> (__ffs(group) - 1) : 0;
      r.groups = (int32_t)groups;
      r.lead = (int32_t)(groups > 0 ? q0 - (c + 1) : at - (c + 1));
      r.tail = (int32_t)(groups > 0 ? at - (q0 + groups * group) : 0);
    }
  }
  constexpr int kFew = 4;
  const int32_t more = r.count();
  if (more > 0 && more <= kFew) {
#pragma unroll 2
    for (int col = lane; col < F; col += 32) {
      float v[kFew + 1];
#pragma unroll
      for (int q = 0; q <= kFew; ++q)
        v[q] = q == 0 ? partial[(c * 2 + 1) * F + col] : q <= more ? partial[r.chunk(q - 1) * 2 * F + col] : 0.0f;
      float s = v[0];
#pragma unroll
      for (int q = 1; q <= kFew; ++q) s += v[q];
      const float f[1] = {scale * s};
      vio::store_stream<TO, 1>(out + (int64_t)key * out_ld + col, f);
    }
  }
  if (lane == 0 && more > kFew) {
    const int at = atomicAdd(&big_runs, 1);
    run[at] = r;
    run_chunk[at] = c;
    run_key[at] = key;
  }
  __syncthreads();
  const int cx = (int)threadIdx.x & (wide - 1), ry = (int)threadIdx.x / wide, rows = kCombineWarps * 32 / wide;
  for (int w = 0; w < big_runs; ++w) {
    const Pieces big = run[w];
    const int32_t m = big.count(), key_w = run_key[w];
    const int64_t cw = run_chunk[w];
    for (int col0 = 0; col0 < F; col0 += wide) {
      const int col = col0 + cx;
      const bool on = col < F;
      float s = ry == 0 && on ? partial[(cw * 2 + 1) * F + col] : 0.0f;
      for (int32_t q = ry; q < m; q += 8 * rows) {
        float v[8];
#pragma unroll
        for (int u = 0; u < 8; ++u) v[u] = on && q + u * rows < m ? partial[big.chunk(q + u * rows) * 2 * F + col] : 0.0f;
#pragma unroll
        for (int u = 0; u < 8; ++u) s += v[u];
      }
      sums[threadIdx.x] = s;
      __syncthreads();
      if (ry == 0 && on) {
        for (int k = 1; k < rows; ++k) s += sums[k * wide + cx];
        const float f[1] = {scale * s};
        vio::store_stream<TO, 1>(out + (int64_t)key_w * out_ld + col, f);
      }
      __syncthreads();
    }
  }
}

// Small plans: one block per run (and 32 * VEC columns); its warps take every so-manieth row, and their sums are added in warp
// order.  A lane asks for one of its warp's next 32 row numbers, so that the rows follow eight at a time without a round
// trip for their numbers.  The first blocks write the zero rows, 32 tokens per warp (4,096 x 128 float32 over 100,000 tokens: 26 us,
// 30 with these blocks last).
// WARPS: 16 where a token has eight rows or more on average, else 8.  In a graph, ordering included: 4,039 x 128 float32 over 301 tokens
// 13.2 us with 16 and 15.7 with 8, 4,096 x 256 bf16 over 4 tokens 21.5 and 28.9; 4,000 x 512 bf16 over 2,000 tokens 34.8
// and 23.6.  (8 warps, each row number asked for on its own: 17.2, 39.3 and 23.1.)
template <typename T, typename TO, int VEC, int WARPS>
__global__ void __launch_bounds__(WARPS * 32) grad_small(const T* __restrict__ dout, int64_t dout_ld, const int32_t* __restrict__ runs,
                                                             const int32_t* __restrict__ keys, const int32_t* __restrict__ idx,
                                                             const uint32_t* __restrict__ present, unsigned zero_blocks, int32_t V,
                                                             int32_t F, float scale, TO* __restrict__ out, int64_t out_ld) {
  __shared__ float sums[WARPS][32 * VEC];
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  const int col = (blockIdx.y * 32 + lane) * VEC;
  const bool on = col < F;
  if (blockIdx.x < zero_blocks) {
    const int64_t v0 = ((int64_t)blockIdx.x * WARPS + warp) * 32;
    if (v0 >= V || !on) return;
    uint32_t gone = ~present[v0 >> 5];
    if (V - v0 < 32) gone &= (1u << (V - v0)) - 1u;
    const vio::Vec<VEC> z(0.0f);
    for (; gone; gone &= gone - 1) vio::store_stream<TO, VEC>(out + (v0 + __ffs(gone) - 1) * out_ld + col, z.v);
    return;
  }
  const int run = (int)(blockIdx.x - zero_blocks);
  if (run >= runs[0]) return;
  const int lo = runs[1 + run], hi = runs[2 + run], v = keys[lo];
  vio::Vec<VEC> acc(0.0f);
  constexpr int U = 8;
  for (int p = lo + warp; p < hi; p += 32 * WARPS) {
    const int left = (hi - p + WARPS - 1) / WARPS; // rows of this warp from here on
    const int mine = lane < left ? idx[p + lane * WARPS] : 0;
    for (int j0 = 0; j0 < 32 && j0 < left; j0 += U) {
      vio::Raw<T, VEC> r[U];
#pragma unroll
      for (int u = 0; u < U; ++u) {
        const int i = __shfl_sync(0xffffffffu, mine, j0 + u);
        if (on && j0 + u < left) r[u].template load<true>(dout + (int64_t)i * dout_ld + col);
        else r[u].zero();
      }
#pragma unroll
      for (int u = 0; u < U; ++u)
#pragma unroll
        for (int e = 0; e < VEC; ++e) acc.v[e] += r[u].get(e);
    }
  }
#pragma unroll
  for (int e = 0; e < VEC; ++e) sums[warp][lane * VEC + e] = acc.v[e];
  __syncthreads();
  if (warp > 0 || !on) return;
#pragma unroll
  for (int w = 1; w < WARPS; ++w)
#pragma unroll
    for (int e = 0; e < VEC; ++e) acc.v[e] += sums[w][lane * VEC + e];
  vio::store_stream<TO, VEC>(out + (int64_t)v * out_ld + col, vio::mul(acc, scale).v);
}

template <typename T, typename TO, int VEC>
int32_t grad_vec(gnnco_handle* h, const PlanLayout& L, const T* dout, int64_t dout_ld, int64_t rows, int32_t V, int32_t F,
                 float scale, TO* out, int64_t out_ld, cudaStream_t st) {
  const int vecs = (F + VEC - 1) / VEC;
  if (is_small(rows)) {
    const unsigned rb = (unsigned)(rows < V ? rows : V);
    auto run = [&](auto kernel, int warps) {
      const unsigned zb = (unsigned)(((int64_t)V + 32 * warps - 1) / (32 * warps));
      kernel<<<dim3(rb + zb, (unsigned)((vecs + 31) / 32)), 32 * warps, 0, st>>>(dout, dout_ld, L.runs, plan_keys(L), plan_rows(L), L.present,
                                                                                 zb, V, F, scale, out, out_ld);
    };
    if (rows >= 8 * (int64_t)V) run(grad_small<T, TO, VEC, 16>, 16);
    else run(grad_small<T, TO, VEC, 8>, 8);
    h->launches += 1;
    GNNCO_LAUNCH_CHECK();
    return GNNCO_OK;
  }
  const int team = vecs <= 8 ? 8 : vecs <= 16 ? 16 : 32;
  const int teams = 256 / team;
  const unsigned cb = (unsigned)((L.chunks + teams - 1) / teams);
  const int32_t *keys = plan_keys(L), *idx = plan_rows(L);
  if (L.chunks > 0) {
    constexpr int K = VEC == 1 ? 4 : VEC == 2 ? 2 : 1;
    const unsigned mb = (unsigned)((rows + 256 * kMarkPer - 1) / (256 * kMarkPer));
#define GNNCO_GRAD(TM, KK)                                                                                                        \
  grad_chunks<T, TO, VEC, TM, KK><<<dim3(cb + mb, (unsigned)((vecs + TM * KK - 1) / (TM * KK))), 256, 0, st>>>(                   \
      dout, dout_ld, keys, idx, rows, V, F, scale, L.chunk, L.chunks, cb, L.present, L.partial, out, out_ld)
    if (team == 8) GNNCO_GRAD(8, 1);
    else if (team == 16) GNNCO_GRAD(16, 1);
    else if (vecs <= 32) GNNCO_GRAD(32, 1);
    else GNNCO_GRAD(32, K);
#undef GNNCO_GRAD
    h->launches += 1;
  }
  const unsigned pb = (unsigned)((L.chunks + kCombineWarps - 1) / kCombineWarps);
  const unsigned zb = (unsigned)(((int64_t)V + 32 * kCombineWarps - 1) / (32 * kCombineWarps));
  int wide = 32;
  while (wide < 256 && wide < F) wide *= 2;
  const bool vec4 = F % 4 == 0 && vec_ok(out, out_ld, sizeof(TO), 4);
  grad_combine<TO><<<pb + zb, kCombineWarps * 32, 0, st>>>(keys, rows, V, F, scale, L.chunk, L.chunks, teams, wide, vec4, pb, L.present,
                                                         L.partial, out, out_ld);
  h->launches += 1;
  GNNCO_LAUNCH_CHECK();
  return GNNCO_OK;
}

template <typename T, typename TO>
int32_t grad_typed(gnnco_handle* h, const PlanLayout& L, const void* dout, int64_t dout_ld, int64_t rows, int32_t V, int32_t F,
                   float scale, void* out, int64_t out_ld, cudaStream_t st) {
  auto fits = [&](int vec) {
    return F % vec == 0 && vec_ok(dout, dout_ld, sizeof(T), vec) && vec_ok(out, out_ld, sizeof(TO), vec);
  };
  const T* d = static_cast<const T*>(dout);
  TO* o = static_cast<TO*>(out);
  if (sizeof(T) == 2 && fits(8)) return grad_vec<T, TO, 8>(h, L, d, dout_ld, rows, V, F, scale, o, out_ld, st);
  if (fits(4)) return grad_vec<T, TO, 4>(h, L, d, dout_ld, rows, V, F, scale, o, out_ld, st);
  if (fits(2)) return grad_vec<T, TO, 2>(h, L, d, dout_ld, rows, V, F, scale, o, out_ld, st);
  return grad_vec<T, TO, 1>(h, L, d, dout_ld, rows, V, F, scale, o, out_ld, st);
}

bool valid_table(int64_t rows, int32_t V, int32_t F) {
  return rows >= 0 && rows < ((int64_t)1 << 31) - 1 && V >= 1 && V < INT32_MAX && F >= 1 && F <= 65536;
}

}  // namespace

extern "C" int32_t gnnco_embedding_lookup(gnnco_handle* h, int32_t table_dtype, int32_t out_dtype, int64_t rows, int32_t V,
                                          int32_t F, const int32_t* tokens, const void* table, int64_t table_ld, float scale,
                                          void* out, int64_t out_ld, void* stream) {
  if (!h || !table || !valid_table(rows, V, F) || table_ld < F || out_ld < F) return GNNCO_INVALID_ARGUMENT;
  if (rows > 0 && (!tokens || !out)) return GNNCO_INVALID_ARGUMENT;
  if ((table_dtype != GNNCO_F32 && table_dtype != GNNCO_BF16) || (out_dtype != GNNCO_F32 && out_dtype != GNNCO_BF16))
    return GNNCO_UNSUPPORTED;
  if (rows == 0) return GNNCO_OK;
  cudaStream_t st = static_cast<cudaStream_t>(stream);
  ProfScope prof_(h, K_EMBED, st);
  typedef __nv_bfloat16 B;
  if (table_dtype == GNNCO_F32 && out_dtype == GNNCO_F32)
    return lookup_typed(h, tokens, (const float*)table, table_ld, (float*)out, out_ld, rows, V, F, scale, st);
  if (table_dtype == GNNCO_F32)
    return lookup_typed(h, tokens, (const float*)table, table_ld, (B*)out, out_ld, rows, V, F, scale, st);
  if (out_dtype == GNNCO_F32)
    return lookup_typed(h, tokens, (const B*)table, table_ld, (float*)out, out_ld, rows, V, F, scale, st);
  return lookup_typed(h, tokens, (const B*)table, table_ld, (B*)out, out_ld, rows, V, F, scale, st);
}

extern "C" int32_t gnnco_embedding_plan_bytes(int64_t rows, int32_t V, int32_t F, size_t* bytes) {
  if (!bytes || !valid_table(rows, V, F)) return GNNCO_INVALID_ARGUMENT;
  *bytes = plan_layout(nullptr, rows, V, F).bytes;
  return GNNCO_OK;
}

extern "C" int32_t gnnco_embedding_plan(gnnco_handle* h, const int32_t* tokens, int64_t rows, int32_t V, int32_t F, void* plan_ws,
                                        size_t plan_bytes, void* stream) {
  if (!h || !plan_ws || ((uintptr_t)plan_ws & 255) || !valid_table(rows, V, F) || (rows > 0 && !tokens))
    return GNNCO_INVALID_ARGUMENT;
  const PlanLayout L = plan_layout(plan_ws, rows, V, F);
  if (plan_bytes < L.bytes) return GNNCO_WORKSPACE_TOO_SMALL;
  cudaStream_t st = static_cast<cudaStream_t>(stream);
  ProfScope prof_(h, K_EMBED, st);
  if (is_small(rows)) {
    const bool clear = V <= (1 << 18);                     // the block clears up to 8,192 words itself
    if (!clear) GNNCO_CUDA_TRY(cudaMemsetAsync(L.present, 0, ((size_t)V + 31) / 32 * 4, st));
    order_small<<<1, kSmallThreads, 0, st>>>(tokens, (int32_t)rows, V, bits_of(V), const_cast<int32_t*>(plan_keys(L)),
                                             const_cast<int32_t*>(plan_rows(L)), L.present, clear, L.runs, h->status);
    h->launches += 1;
    GNNCO_LAUNCH_CHECK();
    return GNNCO_OK;
  }
  if (rows == 0) {
    GNNCO_CUDA_TRY(cudaMemsetAsync(L.present, 0, ((size_t)V + 31) / 32 * 4, st));
    return GNNCO_OK;
  }
  static std::atomic<int> allowed_first{0}, allowed_rest{0};
  int32_t rc = allow_shared_memory(order_scatter<true>, kScatterSmem, h->device, allowed_first);
  if (rc == GNNCO_OK) rc = allow_shared_memory(order_scatter<false>, kScatterSmem, h->device, allowed_rest);
  if (rc != GNNCO_OK) return rc;
  const int64_t tiles = (rows + kOrdTile - 1) / kOrdTile;
  const int64_t per = (tiles + kOrdMaxBlocks - 1) / kOrdMaxBlocks;
  const int64_t span = per * kOrdTile;
  const int nb = (int)((rows + span - 1) / span), digits = 1 << L.bits;
  int32_t *ka = L.key_a, *ia = L.idx_a, *kb = L.key_b, *ib = L.idx_b;
  const int32_t* kin = tokens;
  const int32_t* iin = nullptr;
  for (int p = 0; p < L.passes; ++p) {
    const int shift = p * L.bits;
    if (p == 0) order_histogram<true><<<nb, kOrdThreads, 0, st>>>(kin, rows, span, shift, digits, V, L.hist, L.present, h->status);
    else order_histogram<false><<<nb, kOrdThreads, 0, st>>>(kin, rows, span, shift, digits, V, L.hist, nullptr, nullptr);
    // few blocks: the scatter adds up the block counts itself
    const bool scanned = nb > kOrdFewBlocks;
    if (scanned) order_scan<<<digits, (nb + 31) / 32 * 32, 0, st>>>(L.hist, L.totals, nb);
    if (p == 0)
      order_scatter<true><<<nb, kOrdThreads, kScatterSmem, st>>>(kin, iin, ka, ia, (uint32_t)rows, (uint32_t)span, shift, L.bits, V, L.hist,
                                                                scanned ? L.totals : nullptr);
    else
      order_scatter<false><<<nb, kOrdThreads, kScatterSmem, st>>>(kin, iin, ka, ia, (uint32_t)rows, (uint32_t)span, shift, L.bits, V, L.hist,
                                                                 scanned ? L.totals : nullptr);
    kin = ka; iin = ia;
    int32_t* t = ka; ka = kb; kb = t;
    t = ia; ia = ib; ib = t;
    h->launches += scanned ? 3 : 2;
  }
  GNNCO_LAUNCH_CHECK();
  return GNNCO_OK;
}

extern "C" int32_t gnnco_embedding_grad(gnnco_handle* h, int32_t grad_dtype, int32_t table_dtype, int64_t rows, int32_t V, int32_t F,
                                        const void* dout, int64_t dout_ld, float scale, void* plan_ws, size_t plan_bytes,
                                        void* dtable, int64_t dtable_ld, void* stream) {
  if (!h || !plan_ws || ((uintptr_t)plan_ws & 255) || !dtable || !valid_table(rows, V, F) || dout_ld < F || dtable_ld < F)
    return GNNCO_INVALID_ARGUMENT;
  if (rows > 0 && !dout) return GNNCO_INVALID_ARGUMENT;
  if ((grad_dtype != GNNCO_F32 && grad_dtype != GNNCO_BF16) || (table_dtype != GNNCO_F32 && table_dtype != GNNCO_BF16))
    return GNNCO_UNSUPPORTED;
  const PlanLayout L = plan_layout(plan_ws, rows, V, F);
  if (plan_bytes < L.bytes) return GNNCO_WORKSPACE_TOO_SMALL;
  cudaStream_t st = static_cast<cudaStream_t>(stream);
  ProfScope prof_(h, K_EMBED, st);
  typedef __nv_bfloat16 B;
  if (grad_dtype == GNNCO_F32 && table_dtype == GNNCO_F32)
    return grad_typed<float, float>(h, L, dout, dout_ld, rows, V, F, scale, dtable, dtable_ld, st);
  if (grad_dtype == GNNCO_F32) return grad_typed<float, B>(h, L, dout, dout_ld, rows, V, F, scale, dtable, dtable_ld, st);
  if (table_dtype == GNNCO_F32) return grad_typed<B, float>(h, L, dout, dout_ld, rows, V, F, scale, dtable, dtable_ld, st);
  return grad_typed<B, B>(h, L, dout, dout_ld, rows, V, F, scale, dtable, dtable_ld, st);
}
