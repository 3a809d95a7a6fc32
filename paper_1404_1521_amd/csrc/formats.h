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

}  // namespace pg
