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
#include "internal.cuh"
#include "vec_io.cuh"

namespace {

// -------------------------------------------------------------------------------------------------------- lookup

// A warp owns a tile of `tile` rows; its lanes walk the tile's vectors as one flat list, so that any width keeps all
// lanes busy, and eight loads are in flight per lane.  32-row tiles read the tokens in one coalesced load; calls with
// few rows use 4-row tiles to spread over the SMs.
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
      float f[VEC];
#pragma unroll
      for (int e = 0; e < VEC; ++e) f[e] = scale * v[k].get(e);
      vio::store_stream<TO, VEC>(out + (row0 + r[k]) * out_ld + (int64_t)j[k] * VEC, f);
    }
  }
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
    lookup_kernel<TT, TO, 8><<<grid, 256, 0, st>>>(tokens, table, table_ld, out, out_ld, rows, V, F / 8, scale, tile, h->status);
  else if (fits(4))
    lookup_kernel<TT, TO, 4><<<grid, 256, 0, st>>>(tokens, table, table_ld, out, out_ld, rows, V, F / 4, scale, tile, h->status);
  else
    lookup_kernel<TT, TO, 1><<<grid, 256, 0, st>>>(tokens, table, table_ld, out, out_ld, rows, V, F, scale, tile, h->status);
  h->launches += 1;
  GNNCO_LAUNCH_CHECK();
  return GNNCO_OK;
}

// ---------------------------------------------------------------------------------------------------- order by token
//
// Stable least-significant-digit radix sort of the row numbers by token, 8 bits per pass, only as many passes as V has
// bits.  A fixed number of blocks owns one contiguous span of positions each: block histograms (digit-major), one
// block per digit scans that digit's row, and the scatter turns (digit total, row prefix) into output positions.
// Rows without a token get key V and end up last.  `present` receives one bit per token that occurs.
constexpr int kOrdThreads = 256, kOrdWarps = kOrdThreads / 32, kOrdRounds = 8;
constexpr int kOrdTile = kOrdThreads * kOrdRounds;         // positions of one block-wide step
constexpr int kOrdMaxBlocks = 592;
constexpr int kSmallRows = 4096;                           // up to here one block sorts everything in shared memory

struct PlanLayout {
  int32_t *key_a, *idx_a, *key_b, *idx_b, *hist, *totals;
  uint32_t* present;
  float* partial;                                          // [chunks][2][F]
  size_t bytes;
  int64_t chunks;
  int chunk;
  int passes;
};

int bits_of(int64_t x) {                                   // bits needed for values 0 .. x
  int b = 0;
  while (((int64_t)1 << b) <= x) ++b;
  return b;
}

// Positions of one chunk of the gradient: enough chunks to fill the GPU, at most 256 so that a token's partial sums
// stay few, at least 16 so that the chunk boundaries (a partial row each) do not outweigh the rows.
int chunk_of(int64_t rows) {
  int c = 16;
  while (c < 256 && rows / (2 * c) >= 148 * 32) c *= 2;
  return c;
}

PlanLayout plan_layout(void* ws, int64_t rows, int32_t V, int32_t F) {
  Carver c(ws, 0);
  PlanLayout L;
  L.passes = (bits_of(V) + 7) / 8;
  L.chunk = chunk_of(rows);
  L.chunks = (rows + L.chunk - 1) / L.chunk;
  L.key_a = c.take<int32_t>(rows);
  L.idx_a = c.take<int32_t>(rows);
  L.key_b = c.take<int32_t>(rows);
  L.idx_b = c.take<int32_t>(rows);
  L.hist = c.take<int32_t>(256 * (size_t)kOrdMaxBlocks);
  L.totals = c.take<int32_t>(256);
  L.present = c.take<uint32_t>(((size_t)V + 31) / 32);
  L.partial = c.take<float>((size_t)L.chunks * 2 * F);
  L.bytes = c.off;
  return L;
}
// the buffers that hold the result after `passes` passes
const int32_t* plan_keys(const PlanLayout& L) { return (L.passes & 1) ? L.key_a : L.key_b; }
const int32_t* plan_rows(const PlanLayout& L) { return (L.passes & 1) ? L.idx_a : L.idx_b; }

__device__ __forceinline__ int32_t token_key(int32_t t, int32_t V) { return (uint32_t)t < (uint32_t)V ? t : V; }

// FIRST: keys come from the token vector (row number = position); tokens are checked and marked present.
template <bool FIRST>
__global__ void __launch_bounds__(kOrdThreads) order_histogram(const int32_t* __restrict__ keys, int64_t N, int64_t span,
                                                               int shift, int32_t V, int32_t* __restrict__ hist,
                                                               uint32_t* present, int32_t* status) {
  __shared__ int32_t cnt[256];
  cnt[threadIdx.x] = 0;
  __syncthreads();
  const int64_t lo = (int64_t)blockIdx.x * span, hi = min(N, lo + span);
  for (int64_t p0 = lo; p0 < hi; p0 += kOrdThreads * 4) {
    int32_t k[4];
#pragma unroll
    for (int u = 0; u < 4; ++u) {
      const int64_t p = p0 + u * kOrdThreads + threadIdx.x;
      k[u] = p < hi ? keys[p] : -2;
    }
#pragma unroll
    for (int u = 0; u < 4; ++u) {
      const int64_t p = p0 + u * kOrdThreads + threadIdx.x;
      if (p >= hi) continue;
      if (FIRST) {
        if (k[u] >= V) atomicMin(status, (int32_t)GNNCO_OUT_OF_RANGE);
        k[u] = token_key(k[u], V);
        if (k[u] < V) {
          const uint32_t bit = 1u << (k[u] & 31);
          volatile uint32_t* word = present + (k[u] >> 5);
          if (!(*word & bit)) atomicOr(present + (k[u] >> 5), bit);   // most rows find their bit set already
        }
      }
      atomicAdd(&cnt[(k[u] >> shift) & 255], 1);
    }
  }
  __syncthreads();
  hist[(int64_t)threadIdx.x * gridDim.x + blockIdx.x] = cnt[threadIdx.x];
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

// exclusive prefix over 256 values, one per thread of a 256-thread block
__device__ __forceinline__ int32_t scan256(int32_t x, int32_t* warp_tot) {
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
  for (int w = 0; w < 8; ++w)
    if (w < warp) off += warp_tot[w];
  return off + incl - x;
}

template <bool FIRST>
__global__ void __launch_bounds__(kOrdThreads) order_scatter(const int32_t* __restrict__ keys, const int32_t* __restrict__ idx,
                                                             int32_t* __restrict__ keys_out, int32_t* __restrict__ idx_out,
                                                             int64_t N, int64_t span, int shift, int32_t V,
                                                             const int32_t* __restrict__ hist, const int32_t* __restrict__ totals) {
  __shared__ int32_t cnt[kOrdWarps][256];
  __shared__ int32_t next[256];
  __shared__ int32_t warp_tot[8];
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  const int32_t base = scan256(totals[threadIdx.x], warp_tot);
  next[threadIdx.x] = base + hist[(int64_t)threadIdx.x * gridDim.x + blockIdx.x];
  const int64_t lo = (int64_t)blockIdx.x * span, hi = min(N, lo + span);
  for (int64_t p0 = lo; p0 < hi; p0 += kOrdTile) {
#pragma unroll
    for (int w = 0; w < kOrdWarps; ++w) cnt[w][threadIdx.x] = 0;
    __syncthreads();
    // ranks inside the warp's 256 consecutive positions, in position order
    int32_t k[kOrdRounds], v[kOrdRounds];
    int rank[kOrdRounds];
    const int64_t wbase = p0 + warp * (32 * kOrdRounds);
#pragma unroll
    for (int r = 0; r < kOrdRounds; ++r) {
      const int64_t p = wbase + r * 32 + lane;
      k[r] = p < hi ? (FIRST ? token_key(keys[p], V) : keys[p]) : 0;
      v[r] = FIRST ? (int32_t)p : (p < hi ? idx[p] : 0);
    }
#pragma unroll
    for (int r = 0; r < kOrdRounds; ++r) {
      const bool valid = wbase + r * 32 + lane < hi;
      const uint32_t d = valid ? (uint32_t)(k[r] >> shift) & 255u : 256u;
      const uint32_t peers = __match_any_sync(0xffffffffu, d);
      const int before = __popc(peers & ((1u << lane) - 1u));
      rank[r] = valid ? cnt[warp][d] + before : 0;
      __syncwarp();
      if (valid && before == 0) cnt[warp][d] += __popc(peers);
      __syncwarp();
    }
    __syncthreads();
    {
      int32_t at = next[threadIdx.x];
#pragma unroll
      for (int w = 0; w < kOrdWarps; ++w) {
        const int32_t c = cnt[w][threadIdx.x];
        cnt[w][threadIdx.x] = at;
        at += c;
      }
      next[threadIdx.x] = at;
    }
    __syncthreads();
#pragma unroll
    for (int r = 0; r < kOrdRounds; ++r) {
      if (wbase + r * 32 + lane < hi) {
        const int32_t at = cnt[warp][(k[r] >> shift) & 255] + rank[r];
        keys_out[at] = k[r];
        idx_out[at] = v[r];
      }
    }
    __syncthreads();
  }
}

// All passes in one block for up to kSmallRows rows: 32 warps x 128 positions.
constexpr int kSmallThreads = 1024, kSmallRounds = kSmallRows / kSmallThreads;
constexpr size_t kSmallSmem = (size_t)kSmallRows * 8 + 32 * 256 * 4;
__global__ void __launch_bounds__(kSmallThreads) order_small(const int32_t* __restrict__ tokens, int32_t N, int32_t V, int passes,
                                                             int32_t* __restrict__ keys_out, int32_t* __restrict__ idx_out,
                                                             uint32_t* present, int32_t* status) {
  extern __shared__ int32_t sm[];
  int32_t* sk = sm;
  int32_t* si = sm + kSmallRows;
  int32_t(*cnt)[256] = reinterpret_cast<int32_t(*)[256]>(sm + 2 * kSmallRows);
  __shared__ int32_t warp_tot[8];
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  for (int w = threadIdx.x; w < (V + 31) / 32; w += kSmallThreads) present[w] = 0u;
  __syncthreads();
  int32_t k[kSmallRounds], v[kSmallRounds];
  const int wbase = warp * (32 * kSmallRounds);
#pragma unroll
  for (int r = 0; r < kSmallRounds; ++r) {
    const int p = wbase + r * 32 + lane;
    const int32_t t = p < N ? tokens[p] : -1;
    if (t >= V) atomicMin(status, (int32_t)GNNCO_OUT_OF_RANGE);
    k[r] = token_key(t, V);
    v[r] = p;
    if (p < N && k[r] < V) atomicOr(present + (k[r] >> 5), 1u << (k[r] & 31));
  }
  for (int pass = 0; pass < passes; ++pass) {
    const int shift = 8 * pass;
    for (int q = threadIdx.x; q < 32 * 256; q += kSmallThreads) (&cnt[0][0])[q] = 0;
    __syncthreads();
    int rank[kSmallRounds];
#pragma unroll
    for (int r = 0; r < kSmallRounds; ++r) {
      const bool valid = wbase + r * 32 + lane < N;
      const uint32_t d = valid ? (uint32_t)(k[r] >> shift) & 255u : 256u;
      const uint32_t peers = __match_any_sync(0xffffffffu, d);
      const int before = __popc(peers & ((1u << lane) - 1u));
      rank[r] = valid ? cnt[warp][d] + before : 0;
      __syncwarp();
      if (valid && before == 0) cnt[warp][d] += __popc(peers);
      __syncwarp();
    }
    __syncthreads();
    // digit totals, their prefix, then the per-warp starts
    int32_t total = 0;
    if (threadIdx.x < 256)
      for (int w = 0; w < 32; ++w) total += cnt[w][threadIdx.x];
    int32_t incl = total;
#pragma unroll
    for (int d = 1; d < 32; d <<= 1) {
      const int32_t o = __shfl_up_sync(0xffffffffu, incl, d);
      if (lane >= d) incl += o;
    }
    if (threadIdx.x < 256 && lane == 31) warp_tot[warp] = incl;
    __syncthreads();
    if (threadIdx.x < 256) {
      int32_t at = incl - total;
      for (int w = 0; w < warp; ++w) at += warp_tot[w];
      for (int w = 0; w < 32; ++w) {
        const int32_t c = cnt[w][threadIdx.x];
        cnt[w][threadIdx.x] = at;
        at += c;
      }
    }
    __syncthreads();
#pragma unroll
    for (int r = 0; r < kSmallRounds; ++r) {
      if (wbase + r * 32 + lane < N) {
        const int at = cnt[warp][(k[r] >> shift) & 255] + rank[r];
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
    __syncthreads();
  }
#pragma unroll
  for (int r = 0; r < kSmallRounds; ++r) {
    const int p = wbase + r * 32 + lane;
    if (p < N) {
      keys_out[p] = k[r];
      idx_out[p] = v[r];
    }
  }
}

// ------------------------------------------------------------------------------------------------------ gradient
//
// The sorted positions are cut into chunks of equal length, one team of TEAM lanes per chunk and block of TEAM * VEC
// columns, so a token that holds a third of all rows costs no more than a thousand small ones.  A run that lies inside a
// chunk goes straight to the table; the pieces of a run that crosses a chunk boundary meet in `partial`:
// slot 0 = the chunk's first run, begun in an earlier chunk; slot 1 = its last run, begun here and continued in the next.
// The blocks after the last chunk write the zero rows of tokens that do not occur.
template <typename T, typename TO, int VEC, int TEAM>
__global__ void __launch_bounds__(256) grad_chunks(const T* __restrict__ dout, int64_t dout_ld, const int32_t* __restrict__ keys,
                                                   const int32_t* __restrict__ idx, int64_t N, int32_t V, int32_t F, float scale,
                                                   int chunk, int64_t chunks, unsigned chunk_blocks,
                                                   const uint32_t* __restrict__ present, float* __restrict__ partial,
                                                   TO* __restrict__ out, int64_t out_ld) {
  constexpr int TEAMS = 256 / TEAM;
  constexpr int U = VEC >= 8 ? 8 : 16;
  const int tl = threadIdx.x % TEAM, team = threadIdx.x / TEAM;
  const int col = (blockIdx.y * TEAM + tl) * VEC;
  const bool on = col < F;
  if (blockIdx.x >= chunk_blocks) {
    const int64_t v0 = ((int64_t)(blockIdx.x - chunk_blocks) * TEAMS + team) * 32;
    if (v0 >= V || !on) return;
    uint32_t gone = ~present[v0 >> 5];
    if (V - v0 < 32) gone &= (1u << (V - v0)) - 1u;
    float z[VEC];
#pragma unroll
    for (int e = 0; e < VEC; ++e) z[e] = 0.0f;
    while (gone) {
      const int b = __ffs(gone) - 1;
      gone &= gone - 1;
      vio::store_stream<TO, VEC>(out + (v0 + b) * out_ld + col, z);
    }
    return;
  }
  const int64_t c = (int64_t)blockIdx.x * TEAMS + team;
  if (c >= chunks) return;                                 // whole teams leave together (shuffles below name the team)
  const uint32_t mask = TEAM == 32 ? 0xffffffffu : ((1u << TEAM) - 1u) << ((threadIdx.x & 31) / TEAM * TEAM);
  const int64_t p0 = c * chunk, p1 = min(N, p0 + chunk);
  float acc[VEC];
#pragma unroll
  for (int e = 0; e < VEC; ++e) acc[e] = 0.0f;
  int32_t cur = keys[p0];
  bool head = p0 > 0 && keys[p0 - 1] == cur;
  auto to_table = [&]() {
    float f[VEC];
#pragma unroll
    for (int e = 0; e < VEC; ++e) f[e] = scale * acc[e];
    vio::store_stream<TO, VEC>(out + (int64_t)cur * out_ld + col, f);
  };
  auto to_partial = [&](int slot) {
    float* p = partial + (c * 2 + slot) * F + col;
#pragma unroll
    for (int e = 0; e < VEC; ++e) p[e] = acc[e];
  };
  for (int64_t pb = p0; pb < p1 && cur < V; pb += TEAM) {
    const int64_t mine = pb + tl;
    const int32_t k_l = mine < p1 ? keys[mine] : V;
    const int32_t i_l = mine < p1 ? idx[mine] : 0;
#pragma unroll
    for (int j0 = 0; j0 < TEAM; j0 += (U < TEAM ? U : TEAM)) {
      constexpr int UU = U < TEAM ? U : TEAM;
      vio::Raw<T, VEC> v[UU];
      int32_t k[UU];
#pragma unroll
      for (int u = 0; u < UU; ++u) {
        k[u] = __shfl_sync(mask, k_l, j0 + u, TEAM);
        const int32_t i = __shfl_sync(mask, i_l, j0 + u, TEAM);
        if (on && k[u] < V) v[u].template load<true>(dout + (int64_t)i * dout_ld + col);
        else v[u].zero();
      }
#pragma unroll
      for (int u = 0; u < UU; ++u) {
        if (k[u] != cur) {                                 // uniform over the team
          if (cur < V && on && pb + j0 + u < p1) {
            if (head) to_partial(0);
            else to_table();
          }
          if (pb + j0 + u < p1) {
            head = false;
            cur = k[u];
#pragma unroll
            for (int e = 0; e < VEC; ++e) acc[e] = 0.0f;
          }
        }
#pragma unroll
        for (int e = 0; e < VEC; ++e) acc[e] += v[u].get(e);
      }
    }
  }
  if (cur >= V || !on) return;
  const bool goes_on = p1 < N && keys[p1] == cur;
  if (head) to_partial(0);
  else if (goes_on) to_partial(1);
  else to_table();
}

// Runs that cross chunk boundaries: warp w of the block looks at chunk c0 + w; where a run begins there that continues,
// the run's pieces are slot 1 of chunk c and slot 0 of the following chunks.  Few pieces are added by the warp, in chunk
// order; many (a token with thousands of rows) by all warps of the block, each every 32nd piece, and the 32 sums in
// warp order.  Grid.y covers the columns, 32 per block.
constexpr int kCombineWarps = 32;
template <typename TO>
__global__ void __launch_bounds__(kCombineWarps * 32) grad_combine(const int32_t* __restrict__ keys, int64_t N, int32_t V, int32_t F,
                                                                   float scale, int chunk, int64_t chunks,
                                                                   const float* __restrict__ partial, TO* __restrict__ out,
                                                                   int64_t out_ld) {
  __shared__ int32_t big_run[kCombineWarps];               // pieces after the first, 0: nothing to do for the block
  __shared__ float sums[kCombineWarps][33];
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  const int64_t c0 = (int64_t)blockIdx.x * kCombineWarps, c = c0 + warp;
  const int col = blockIdx.y * 32 + lane;
  const bool on = col < F;
  int32_t more = 0, key = V;
  if (c < chunks) {
    const int64_t p0 = c * chunk, p1 = min(N, p0 + chunk);
    key = keys[p1 - 1];
    if (key < V && p1 < N && keys[p1] == key && !(keys[p0] == key && p0 > 0 && keys[p0 - 1] == key)) {
      for (int64_t b = c + 1; b < chunks; b += 32) {
        const bool same = b + lane < chunks && keys[(b + lane) * chunk] == key;
        const uint32_t m = __ballot_sync(0xffffffffu, same);
        more += m == 0xffffffffu ? 32 : __ffs(~m) - 1;
        if (m != 0xffffffffu) break;
      }
    }
  }
  constexpr int kFew = 64;
  if (more > 0 && more <= kFew && on) {
    float s = partial[(c * 2 + 1) * F + col];
    int32_t q = 1;
    for (; q + 7 <= more; q += 8) {
      float v[8];
#pragma unroll
      for (int u = 0; u < 8; ++u) v[u] = partial[(c + q + u) * 2 * F + col];
#pragma unroll
      for (int u = 0; u < 8; ++u) s += v[u];
    }
    for (; q <= more; ++q) s += partial[(c + q) * 2 * F + col];
    float f[1] = {scale * s};
    vio::store_stream<TO, 1>(out + (int64_t)key * out_ld + col, f);
  }
  if (lane == 0) big_run[warp] = more > kFew ? more : 0;
  __syncthreads();
  for (int w = 0; w < kCombineWarps; ++w) {
    const int32_t m = big_run[w];
    if (m == 0) continue;
    const int64_t cw = c0 + w;
    float s = warp == 0 && on ? partial[(cw * 2 + 1) * F + col] : 0.0f;
    int32_t q = 1 + warp;
    for (; q + 7 * kCombineWarps <= m; q += 8 * kCombineWarps) {
      float v[8];
#pragma unroll
      for (int u = 0; u < 8; ++u) v[u] = on ? partial[(cw + q + u * kCombineWarps) * 2 * F + col] : 0.0f;
#pragma unroll
      for (int u = 0; u < 8; ++u) s += v[u];
    }
    for (; q <= m; q += kCombineWarps) s += on ? partial[(cw + q) * 2 * F + col] : 0.0f;
    sums[warp][lane] = s;
    __syncthreads();
    if (warp == 0 && on) {
      float t = 0.0f;
#pragma unroll
      for (int k = 0; k < kCombineWarps; ++k) t += sums[k][lane];
      const int32_t key_w = keys[min(N, cw * chunk + chunk) - 1];
      float f[1] = {scale * t};
      vio::store_stream<TO, 1>(out + (int64_t)key_w * out_ld + col, f);
    }
    __syncthreads();
  }
}

template <typename T, typename TO, int VEC>
int32_t grad_vec(gnnco_handle* h, const PlanLayout& L, const T* dout, int64_t dout_ld, int64_t rows, int32_t V, int32_t F,
                 float scale, TO* out, int64_t out_ld, cudaStream_t st) {
  const int vecs = (F + VEC - 1) / VEC;
  const int team = vecs <= 8 ? 8 : vecs <= 16 ? 16 : 32;
  const int teams = 256 / team;
  const unsigned cb = (unsigned)((L.chunks + teams - 1) / teams);
  const unsigned zb = (unsigned)(((int64_t)(V + 31) / 32 + teams - 1) / teams);
  const dim3 grid(cb + zb, (unsigned)((vecs + team - 1) / team));
  const int32_t *keys = plan_keys(L), *idx = plan_rows(L);
#define GNNCO_GRAD(TM)                                                                                                     \
  grad_chunks<T, TO, VEC, TM><<<grid, 256, 0, st>>>(dout, dout_ld, keys, idx, rows, V, F, scale, L.chunk, L.chunks, cb, \
                                                   L.present, L.partial, out, out_ld)
  if (team == 8) GNNCO_GRAD(8);
  else if (team == 16) GNNCO_GRAD(16);
  else GNNCO_GRAD(32);
#undef GNNCO_GRAD
  h->launches += 1;
  if (L.chunks > 1) {
    grad_combine<TO><<<dim3((unsigned)((L.chunks + kCombineWarps - 1) / kCombineWarps), (unsigned)((F + 31) / 32)),
                       kCombineWarps * 32, 0, st>>>(keys, rows, V, F, scale, L.chunk, L.chunks, L.partial, out, out_ld);
    h->launches += 1;
  }
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
  if (rows > 0 && rows <= kSmallRows) {
    GNNCO_CUDA_TRY(cudaFuncSetAttribute(order_small, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)kSmallSmem));
    order_small<<<1, kSmallThreads, kSmallSmem, st>>>(tokens, (int32_t)rows, V, L.passes, const_cast<int32_t*>(plan_keys(L)),
                                                     const_cast<int32_t*>(plan_rows(L)), L.present, h->status);
    h->launches += 1;
    GNNCO_LAUNCH_CHECK();
    return GNNCO_OK;
  }
  GNNCO_CUDA_TRY(cudaMemsetAsync(L.present, 0, ((size_t)V + 31) / 32 * 4, st));
  if (rows == 0) return GNNCO_OK;
  const int64_t tiles = (rows + kOrdTile - 1) / kOrdTile;
  const int64_t per = (tiles + kOrdMaxBlocks - 1) / kOrdMaxBlocks;
  const int64_t span = per * kOrdTile;
  const int nb = (int)((rows + span - 1) / span);
  int32_t *ka = L.key_a, *ia = L.idx_a, *kb = L.key_b, *ib = L.idx_b;
  const int32_t* kin = tokens;
  const int32_t* iin = nullptr;
  for (int p = 0; p < L.passes; ++p) {
    if (p == 0) order_histogram<true><<<nb, kOrdThreads, 0, st>>>(kin, rows, span, 0, V, L.hist, L.present, h->status);
    else order_histogram<false><<<nb, kOrdThreads, 0, st>>>(kin, rows, span, 8 * p, V, L.hist, nullptr, nullptr);
    order_scan<<<256, 1024, 0, st>>>(L.hist, L.totals, nb);
    if (p == 0) order_scatter<true><<<nb, kOrdThreads, 0, st>>>(kin, iin, ka, ia, rows, span, 0, V, L.hist, L.totals);
    else order_scatter<false><<<nb, kOrdThreads, 0, st>>>(kin, iin, ka, ia, rows, span, 8 * p, V, L.hist, L.totals);
    kin = ka; iin = ia;
    int32_t* t = ka; ka = kb; kb = t;
    t = ia; ia = ib; ib = t;
    h->launches += 3;
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
