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
    } else if constexpr (VEC == 2) {
      __stcs(reinterpret_cast<float2*>(p), make_float2(v[0], v[1]));
    } else {
#pragma unroll
      for (int i = 0; i < VEC; ++i) __stcs(p + i, v[i]);
    }
  } else if constexpr (VEC == 8) {
    __stcs(reinterpret_cast<uint4*>(p), make_uint4(pack_bf16(v[0], v[1]), pack_bf16(v[2], v[3]), pack_bf16(v[4], v[5]),
                                                   pack_bf16(v[6], v[7])));
  } else if constexpr (VEC == 4) {
    __stcs(reinterpret_cast<uint2*>(p), make_uint2(pack_bf16(v[0], v[1]), pack_bf16(v[2], v[3])));
  } else if constexpr (VEC == 2) {
    __stcs(reinterpret_cast<uint32_t*>(p), pack_bf16(v[0], v[1]));
  } else {
#pragma unroll
    for (int i = 0; i < VEC; ++i)
      __stcs(reinterpret_cast<unsigned short*>(p) + i, (unsigned short)(pack_bf16(v[i], 0.0f) & 0xffffu));
  }
}

// Element-wise float32 arithmetic on VEC values, two at a time where VEC is even (one instruction per pair).
__device__ __forceinline__ uint64_t pair_of(float x, float y) {
  uint64_t r;
  asm("mov.b64 %0, {%1, %2};" : "=l"(r) : "f"(x), "f"(y));
  return r;
}
__device__ __forceinline__ void unpair(uint64_t v, float& x, float& y) { asm("mov.b64 {%0, %1}, %2;" : "=f"(x), "=f"(y) : "l"(v)); }

template <int VEC>
struct Vec {
  float v[VEC];
  __device__ __forceinline__ Vec() {}
  __device__ __forceinline__ explicit Vec(float x) {
#pragma unroll
    for (int i = 0; i < VEC; ++i) v[i] = x;
  }
  template <typename T>
  __device__ __forceinline__ explicit Vec(const Raw<T, VEC>& r) {
#pragma unroll
    for (int i = 0; i < VEC; ++i) v[i] = r.get(i);
  }
  __device__ __forceinline__ float sum() const {
    float s = v[0];
#pragma unroll
    for (int i = 1; i < VEC; ++i) s += v[i];
    return s;
  }
};
// a b
template <int VEC>
__device__ __forceinline__ Vec<VEC> mul(const Vec<VEC>& a, const Vec<VEC>& b) {
  Vec<VEC> r;
  if constexpr (VEC % 2 == 0) {
#pragma unroll
    for (int i = 0; i < VEC; i += 2) {
      uint64_t d;
      asm("mul.rn.f32x2 %0, %1, %2;" : "=l"(d) : "l"(pair_of(a.v[i], a.v[i + 1])), "l"(pair_of(b.v[i], b.v[i + 1])));
      unpair(d, r.v[i], r.v[i + 1]);
    }
  } else {
#pragma unroll
    for (int i = 0; i < VEC; ++i) r.v[i] = a.v[i] * b.v[i];
  }
  return r;
}
template <int VEC>
__device__ __forceinline__ Vec<VEC> mul(const Vec<VEC>& a, float b) { return mul(a, Vec<VEC>(b)); }
// a b + c
template <int VEC>
__device__ __forceinline__ Vec<VEC> fma(const Vec<VEC>& a, const Vec<VEC>& b, const Vec<VEC>& c) {
  Vec<VEC> r;
  if constexpr (VEC % 2 == 0) {
#pragma unroll
    for (int i = 0; i < VEC; i += 2) {
      uint64_t d;
      asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(d) : "l"(pair_of(a.v[i], a.v[i + 1])), "l"(pair_of(b.v[i], b.v[i + 1])),
          "l"(pair_of(c.v[i], c.v[i + 1])));
      unpair(d, r.v[i], r.v[i + 1]);
    }
  } else {
#pragma unroll
    for (int i = 0; i < VEC; ++i) r.v[i] = fmaf(a.v[i], b.v[i], c.v[i]);
  }
  return r;
}
template <int VEC>
__device__ __forceinline__ Vec<VEC> fma(const Vec<VEC>& a, float b, const Vec<VEC>& c) { return fma(a, Vec<VEC>(b), c); }

}  // namespace vio

// Whether rows of `ld` elements of `es` bytes starting at p can be moved in vectors of `vec` elements.
static inline bool vec_ok(const void* p, int64_t ld, int es, int vec) {
  const int64_t need = (int64_t)vec * es < 16 ? (int64_t)vec * es : 16;
  return ((uintptr_t)p % need) == 0 && (ld * es) % need == 0;
}
