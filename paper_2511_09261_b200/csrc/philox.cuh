// The counter-based generator Philox4x32-10 (Salmon, Moraes, Dror, Shaw: "Parallel random numbers: as easy as 1, 2, 3",
// SC 2011): four 32-bit words as a function of a 128-bit counter and a 64-bit key, with nothing carried from one
// counter to the next.  Dropout masks are words compared with p 2^32: element (r, c) of a [rows x F] tensor takes word
// c % 4 of counter (r * ceil(F / 4) + c / 4, step, layer), so a mask depends neither on the type nor on the strides of the
// tensor nor on which thread asks, and the backward pass draws it again instead of reading it.
#pragma once

#include <stdint.h>

namespace philox {

constexpr uint32_t kMul0 = 0xD2511F53u, kMul1 = 0xCD9E8D57u, kWeyl0 = 0x9E3779B9u, kWeyl1 = 0xBB67AE85u;

// What a launch passes down.  lim = p 2^32 - 1 in 32 bits: an element is kept if its word is above it (where p 2^32 rounds to 0
// nothing is dropped, and no kernel draws words).
struct Mask {
  uint32_t key[20];                   // both words of every round's key: operands from constant memory, no additions per quad
  uint32_t step, layer, lim;
  float scale;                        // 1 / (1 - p)
  const uint32_t* step_dev;           // added to step where given
};
inline void set_seed(Mask* m, uint64_t seed) {
  for (uint32_t r = 0; r < 10; ++r) {
    m->key[2 * r] = (uint32_t)seed + r * kWeyl0;
    m->key[2 * r + 1] = (uint32_t)(seed >> 32) + r * kWeyl1;
  }
}

// The part of the rounds that all counters of a launch share is computed once: the second product of round 1, and, while the upper
// half of the quad's number stays the same, the first product of round 2 (18 products a quad instead of 20).
struct Stream {
  uint32_t hi1, lo1, last_hi, hi2, lo2;
  __device__ __forceinline__ explicit Stream(const Mask& m) {
    const uint32_t step = m.step + (m.step_dev ? *m.step_dev : 0u);
    hi1 = __umulhi(kMul1, step);
    lo1 = kMul1 * step;
    upper(m, 0u);
  }
  __device__ __forceinline__ void upper(const Mask& m, uint32_t q_hi) {
    last_hi = q_hi;
    const uint32_t x0 = hi1 ^ q_hi ^ m.key[0];
    hi2 = __umulhi(kMul0, x0);
    lo2 = kMul0 * x0;
  }
  __device__ __forceinline__ uint4 quad(const Mask& m, uint64_t q) {
    if ((uint32_t)(q >> 32) != last_hi) upper(m, (uint32_t)(q >> 32));
    return rounds(m, (uint32_t)q);
  }
  // quads q .. q + N - 1, N a power of two that divides q
  template <int N>
  __device__ __forceinline__ void quads(const Mask& m, uint64_t q, uint4 (&w)[N]) {
    if ((uint32_t)(q >> 32) != last_hi) upper(m, (uint32_t)(q >> 32));
#pragma unroll
    for (int k = 0; k < N; ++k) w[k] = rounds(m, (uint32_t)q + k);
  }

 private:
  __device__ __forceinline__ uint4 rounds(const Mask& m, uint32_t q_lo) const {
    const uint64_t a = (uint64_t)kMul0 * q_lo;
    uint32_t x2 = (uint32_t)(a >> 32) ^ m.layer ^ m.key[1], x3 = (uint32_t)a;
    const uint64_t b = (uint64_t)kMul1 * x2;
    uint32_t x0 = (uint32_t)(b >> 32) ^ lo1 ^ m.key[2], x1 = (uint32_t)b;
    x2 = hi2 ^ x3 ^ m.key[3];
    x3 = lo2;
#pragma unroll
    for (int round = 2; round < 10; ++round) {
      const uint64_t u = (uint64_t)kMul0 * x0, v = (uint64_t)kMul1 * x2;
      x0 = (uint32_t)(v >> 32) ^ x1 ^ m.key[2 * round];
      x2 = (uint32_t)(u >> 32) ^ x3 ^ m.key[2 * round + 1];
      x1 = (uint32_t)v;
      x3 = (uint32_t)u;
    }
    return make_uint4(x0, x1, x2, x3);
  }
};

}  // namespace philox
