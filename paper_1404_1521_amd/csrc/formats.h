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

// Four elements in a row: 16 bytes of float32 or 8 of a 16-bit format.  VEC: as one
// aligned word; otherwise element by element, the first n of them.
template <class T>
struct Quad {
  uint2 raw;
  __device__ __forceinline__ float get(int i) const {
    const uint32_t w = i < 2 ? raw.x : raw.y;
    return Elem<T>::get(T{(uint16_t)(i & 1 ? w >> 16 : w)});
  }
};
template <>
struct Quad<float> {
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
    q.raw = *reinterpret_cast<const decltype(q.raw)*>(p);
  } else if constexpr (sizeof(T) == 4) {
#pragma unroll
    for (int i = 0; i < 4; ++i) q.raw[i] = i < n ? p[i] : 0.f;
  } else {
    uint32_t h[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) h[i] = i < n ? p[i].bits : 0u;
    q.raw = uint2{h[0] | h[1] << 16, h[2] | h[3] << 16};
  }
  return q;
}

template <class T, bool VEC>
__device__ __forceinline__ void store_quad(T* p, const float (&v)[4], int n) {
  if constexpr (VEC && sizeof(T) == 4) {
    st4(p, f4{v[0], v[1], v[2], v[3]});
  } else if constexpr (VEC) {
    *reinterpret_cast<uint2*>(p) = uint2{put2(v[0], v[1], T{}), put2(v[2], v[3], T{})};
  } else {
#pragma unroll
    for (int i = 0; i < 4; ++i)
      if (i < n) p[i] = Elem<T>::put(settled(v[i]));
  }
}

}  // namespace pg
