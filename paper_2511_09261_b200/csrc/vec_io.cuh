// Vector access to float32 / bfloat16 rows: VEC consecutive elements as float registers.  A vector of VEC elements is
// moved in pieces of at most 16 bytes; the caller guarantees that base and row stride are multiples of
// min(16, VEC * element size) bytes (vec_width picks the VEC for which that holds).
#pragma once

#include <cuda_bf16.h>
#include <stdint.h>

namespace vio {

template <typename T>
struct Is16 { static constexpr bool value = false; };
template <>
struct Is16<__nv_bfloat16> { static constexpr bool value = true; };

__device__ __forceinline__ float bf_lo(uint32_t v) { return __uint_as_float(v << 16); }
__device__ __forceinline__ float bf_hi(uint32_t v) { return __uint_as_float(v & 0xffff0000u); }
// round to nearest even (NaN stays NaN); lo in the low half
__device__ __forceinline__ uint32_t pack_bf16(float lo, float hi) {
  uint32_t r;
  asm("cvt.rn.bf16x2.f32 %0, %1, %2;" : "=r"(r) : "f"(hi), "f"(lo));
  return r;
}

// The raw bits of VEC elements (held packed until they are used, so that bf16 rows cost half the registers).
template <typename T, int VEC>
struct Raw {
  static constexpr int kBytes = VEC * (int)sizeof(T);
  static constexpr int kWords = kBytes >= 4 ? kBytes / 4 : 1;
  uint32_t w[kWords];

  __device__ __forceinline__ void zero() {
#pragma unroll
    for (int i = 0; i < kWords; ++i) w[i] = 0u;
  }
  // STREAM: the line is not needed again (evict first)
  template <bool STREAM>
  __device__ __forceinline__ void load(const T* p) {
    if constexpr (kBytes % 16 == 0) {
#pragma unroll
      for (int i = 0; i < kBytes / 16; ++i) {
        const uint4* q = reinterpret_cast<const uint4*>(p) + i;
        const uint4 v = STREAM ? __ldcs(q) : __ldg(q);
        w[4 * i] = v.x; w[4 * i + 1] = v.y; w[4 * i + 2] = v.z; w[4 * i + 3] = v.w;
      }
    } else if constexpr (kBytes == 8) {
      const uint2* q = reinterpret_cast<const uint2*>(p);
      const uint2 v = STREAM ? __ldcs(q) : __ldg(q);
      w[0] = v.x; w[1] = v.y;
    } else if constexpr (kBytes == 4) {
      const uint32_t* q = reinterpret_cast<const uint32_t*>(p);
      w[0] = STREAM ? __ldcs(q) : __ldg(q);
    } else {
      const unsigned short* q = reinterpret_cast<const unsigned short*>(p);
      w[0] = STREAM ? __ldcs(q) : __ldg(q);
    }
  }
  __device__ __forceinline__ float get(int i) const {
    if constexpr (Is16<T>::value) return (i & 1) ? bf_hi(w[i >> 1]) : bf_lo(w[i >> 1]);
    else return __uint_as_float(w[i]);
  }
};

template <typename T, int VEC>
__device__ __forceinline__ void store_stream(T* p, const float (&v)[VEC]) {
  if constexpr (!Is16<T>::value) {
    if constexpr (VEC % 4 == 0) {
#pragma unroll
      for (int i = 0; i < VEC / 4; ++i)
        __stcs(reinterpret_cast<float4*>(p) + i, make_float4(v[4 * i], v[4 * i + 1], v[4 * i + 2], v[4 * i + 3]));
    } else {
#pragma unroll
      for (int i = 0; i < VEC; ++i) __stcs(p + i, v[i]);
    }
  } else if constexpr (VEC == 8) {
    __stcs(reinterpret_cast<uint4*>(p), make_uint4(pack_bf16(v[0], v[1]), pack_bf16(v[2], v[3]), pack_bf16(v[4], v[5]),
                                                   pack_bf16(v[6], v[7])));
  } else if constexpr (VEC == 4) {
    __stcs(reinterpret_cast<uint2*>(p), make_uint2(pack_bf16(v[0], v[1]), pack_bf16(v[2], v[3])));
  } else {
#pragma unroll
    for (int i = 0; i < VEC; ++i)
      __stcs(reinterpret_cast<unsigned short*>(p) + i, (unsigned short)(pack_bf16(v[i], 0.0f) & 0xffffu));
  }
}

}  // namespace vio

// Whether rows of `ld` elements of `es` bytes starting at p can be moved in vectors of `vec` elements.
static inline bool vec_ok(const void* p, int64_t ld, int es, int vec) {
  const int64_t need = (int64_t)vec * es < 16 ? (int64_t)vec * es : 16;
  return ((uintptr_t)p % need) == 0 && (ld * es) % need == 0;
}
