// Storage formats of tables and tensors, and their conversions to float32.
#pragma once
#include "common.h"

namespace pg {

// Storage formats.  bfloat16 is the upper half of a binary32; rounding a
// float to it keeps the upper half after adding half an ulp minus one plus
// the parity of the kept part (round to nearest, ties to even), and a NaN
// keeps a quiet NaN.  binary16 uses the hardware conversion, which rounds to
// nearest even.
struct BF16 {
  uint16_t bits;
};
struct F16 {
  uint16_t bits;
};

template <class T>
struct Elem;
template <>
struct Elem<float> {
  static __device__ __forceinline__ float get(float v) { return v; }
  static __device__ __forceinline__ float put(float v) { return v; }
};
template <>
struct Elem<BF16> {
  static __device__ __forceinline__ float get(BF16 v) {
    return __uint_as_float((uint32_t)v.bits << 16);
  }
  static __device__ __forceinline__ BF16 put(float f) {
    uint32_t u = __float_as_uint(f);
    if ((u & 0x7fffffffu) > 0x7f800000u) return BF16{(uint16_t)((u >> 16) | 0x40u)};
    u += 0x7fffu + ((u >> 16) & 1u);
    return BF16{(uint16_t)(u >> 16)};
  }
};
template <>
struct Elem<F16> {
  static __device__ __forceinline__ float get(F16 v) {
    return (float)__builtin_bit_cast(_Float16, v.bits);
  }
  static __device__ __forceinline__ F16 put(float f) {
    return F16{__builtin_bit_cast(uint16_t, (_Float16)f)};
  }
};

// Four elements in a row, in one load or store: 16 bytes of float32 or 8 of a
// 16-bit format, aligned to the element only (the hardware takes any address; an
// access that crosses a cache line costs a second one).  Without VEC element by
// element, the first n of them.
typedef float f4_any __attribute__((ext_vector_type(4), aligned(4)));
typedef uint32_t u2_any __attribute__((ext_vector_type(2), aligned(2)));
template <class T>
struct Quad {
  typedef u2_any any;
  u2_any raw;
  __device__ __forceinline__ float get(int i) const {
    const uint32_t w = i < 2 ? raw.x : raw.y;
    return Elem<T>::get(T{(uint16_t)(i & 1 ? w >> 16 : w)});
  }
};
template <>
struct Quad<float> {
  typedef f4_any any;
  f4 raw;
  __device__ __forceinline__ float get(int i) const { return raw[i]; }
};

// A float as it is in its register: what computed it is not fused with what rounds
// it (a fused multiply-add that writes binary16 rounds once where others round twice).
__device__ __forceinline__ float settled(float f) {
  asm("" : "+v"(f));
  return f;
}

// Two floats rounded to a 16-bit format, in the halves of a word.
__device__ __forceinline__ uint32_t put2(float lo, float hi, BF16) {
  typedef __bf16 b2 __attribute__((ext_vector_type(2)));
  return __builtin_bit_cast(uint32_t, b2{(__bf16)lo, (__bf16)hi});
}
__device__ __forceinline__ uint32_t put2(float lo, float hi, F16) {
  typedef _Float16 h2 __attribute__((ext_vector_type(2)));
  return __builtin_bit_cast(uint32_t, h2{(_Float16)settled(lo), (_Float16)settled(hi)});
}

template <class T, bool VEC>
__device__ __forceinline__ Quad<T> load_quad(const T* p, int n) {
  Quad<T> q{};
  if constexpr (VEC) {
    q.raw = *reinterpret_cast<const typename Quad<T>::any*>(p);
  } else if constexpr (sizeof(T) == 4) {
#pragma unroll
    for (int i = 0; i < 4; ++i) q.raw[i] = i < n ? p[i] : 0.f;
  } else {
    uint32_t h[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) h[i] = i < n ? p[i].bits : 0u;
    q.raw = u2_any{h[0] | h[1] << 16, h[2] | h[3] << 16};
  }
  return q;
}

template <class T, bool VEC>
__device__ __forceinline__ void store_quad(T* p, const float (&v)[4], int n) {
  if constexpr (VEC && sizeof(T) == 4) {
    *reinterpret_cast<f4_any*>(p) = f4_any{v[0], v[1], v[2], v[3]};
  } else if constexpr (VEC) {
    *reinterpret_cast<u2_any*>(p) = u2_any{put2(v[0], v[1], T{}), put2(v[2], v[3], T{})};
  } else {
#pragma unroll
    for (int i = 0; i < 4; ++i)
      if (i < n) p[i] = Elem<T>::put(settled(v[i]));
  }
}

// Eight elements in a row, likewise.
typedef uint32_t u4_any __attribute__((ext_vector_type(4), aligned(2)));
template <class T>
struct Oct {
  u4_any raw;
  __device__ __forceinline__ void load(const T* p) { raw = *reinterpret_cast<const u4_any*>(p); }
  __device__ __forceinline__ float get(int i) const {
    const uint32_t w = raw[i / 2];
    return Elem<T>::get(T{(uint16_t)(i & 1 ? w >> 16 : w)});
  }
  static __device__ __forceinline__ void store(T* p, const float (&v)[8]) {
    *reinterpret_cast<u4_any*>(p) = u4_any{put2(v[0], v[1], T{}), put2(v[2], v[3], T{}),
                                           put2(v[4], v[5], T{}), put2(v[6], v[7], T{})};
  }
};
template <>
struct Oct<float> {
  f4_any lo, hi;
  __device__ __forceinline__ void load(const float* p) {
    lo = *reinterpret_cast<const f4_any*>(p);
    hi = *reinterpret_cast<const f4_any*>(p + 4);
  }
  __device__ __forceinline__ float get(int i) const { return i < 4 ? lo[i & 3] : hi[i & 3]; }
  static __device__ __forceinline__ void store(float* p, const float (&v)[8]) {
    *reinterpret_cast<f4_any*>(p) = f4_any{v[0], v[1], v[2], v[3]};
    *reinterpret_cast<f4_any*>(p + 4) = f4_any{v[4], v[5], v[6], v[7]};
  }
};

}  // namespace pg
