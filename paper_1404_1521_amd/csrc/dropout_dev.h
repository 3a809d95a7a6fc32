// Dropout with a mask that is computed and never stored.
//
//   y[r][c] = keep(r, c) ? x[r][c] * scale : 0   (+ add[r][c])
//
// keep compares 16 bits of a counter-based generator with the threshold
// round(65536 p).  Eight columns share one counter, so the generator runs
// once for every eight elements; nothing but x (and add) is read.
#pragma once
#include "formats.h"
#include "operators.h"

namespace pg {

// Philox 4x32-10 (Salmon, Moraes, Dror, Shaw, SC 2011): ten rounds of two
// 32 x 32 -> 64 bit products, the high words mixed with the other counter words
// and a key that grows by a constant (Weyl sequence) each round.
__device__ __forceinline__ uint4 philox10(uint4 c, uint32_t k0, uint32_t k1) {
#pragma unroll
  for (int i = 0; i < 10; ++i) {
    const uint64_t p0 = (uint64_t)0xD2511F53u * c.x, p1 = (uint64_t)0xCD9E8D57u * c.z;
    c = uint4{(uint32_t)(p1 >> 32) ^ c.y ^ k0, (uint32_t)p1, (uint32_t)(p0 >> 32) ^ c.w ^ k1,
              (uint32_t)p0};
    k0 += 0x9E3779B9u;
    k1 += 0xBB67AE85u;
  }
  return c;
}

// Bit j set: element j of the eight is kept.
__device__ __forceinline__ uint32_t keep_bits(uint4 w, uint32_t threshold) {
  uint32_t m = 0;
  const uint32_t v[4] = {w.x, w.y, w.z, w.w};
#pragma unroll
  for (int j = 0; j < 8; ++j)
    m |= ((v[j / 2] >> (16 * (j % 2)) & 0xffffu) >= threshold ? 1u : 0u) << j;
  return m;
}

template <class T>
__global__ __launch_bounds__(kBlock) void k_dropout(DropoutCall c) {
  const polyglot_dropout_args& a = c.a;
  const int groups = (a.d + 7) / 8;
  const int64_t total = a.rows * groups;
  const uint32_t site = a.site + (a.site_dev ? *a.site_dev : 0u);
  for (int64_t i = (int64_t)blockIdx.x * kBlock + threadIdx.x; i < total;
       i += (int64_t)gridDim.x * kBlock) {
    const int64_t r = i / groups;
    const int g = (int)(i - r * groups);
    const uint64_t row = a.first_row + (uint64_t)r;
    const uint4 w = philox10(uint4{a.whole_rows ? 0xffffffffu : (uint32_t)g, (uint32_t)row,
                                   (uint32_t)(row >> 32), site},
                             (uint32_t)a.seed, (uint32_t)(a.seed >> 32));
    uint32_t keep = keep_bits(w, c.threshold);
    if (a.whole_rows) keep = keep & 1u ? 0xffu : 0u;
    int64_t from = r;
    bool bad = false;
    if (a.ids) {
      from = a.id_bytes == 8 ? static_cast<const int64_t*>(a.ids)[r]
                             : static_cast<const int32_t*>(a.ids)[r];
      bad = from < 0 || from >= a.table_rows;
      if (bad) atomicOr(c.flag, kFlagBadId);
    }
    const T* x = static_cast<const T*>(a.x) + (bad ? 0 : from) * a.ld_x;
    const T* add = a.add ? static_cast<const T*>(a.add) + r * a.ld_add : nullptr;
    T* y = static_cast<T*>(a.y) + r * a.ld_y;
    for (int j = 0; j < 8 && g * 8 + j < a.d; ++j) {
      const int col = g * 8 + j;
      float v = keep >> j & 1u ? Elem<T>::get(x[col]) * c.scale : 0.f;
      if (add) v += Elem<T>::get(add[col]);
      y[col] = Elem<T>::put(bad ? __builtin_nanf("") : v);
    }
  }
}

}  // namespace pg
