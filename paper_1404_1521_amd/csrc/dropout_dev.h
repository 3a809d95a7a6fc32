// Dropout with a mask that is computed and never stored.
//
//   y[r][c] = keep(r, c) ? x[r][c] * scale : 0   (+ add[r][c])
//
// keep compares 16 bits of a counter-based generator with the threshold
// round(65536 p).  Eight columns share one counter, so the generator runs once
// for every eight elements; nothing but x (and add) is read.
//
// Bound by memory where the tensors are large, by the launch where they are small:
// 262,144 x 512 float16 95 us (5.7 TB/s read and written), 5,120 gathered rows of 64
// float32 3.4 us.  Widths of other than whole eights are bound by their last columns: the
// loop over them loads after the generator, one element at a time, and nearly every wave
// has a lane in it.  20,011 rows of bfloat16 with an addition: 199 wide 8.0 us, 200 wide 4.9.
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

// The quotient n / groups of a workgroup's places, n < groups + kDropPlaces.
constexpr int kDropPlaces = kBlock;
__device__ __forceinline__ uint32_t rows_down(uint32_t n, const DropoutCall& c) {
  if (c.groups >= kDropPlaces) return n >= (uint32_t)c.groups ? 1u : 0u;
  return c.groups == 1 ? n : __umulhi(n, c.groups_inv);
}

// A workgroup takes 256 consecutive groups of eight columns, counted through all
// rows, so that rows of every width fill its lanes; only the workgroup's first place
// takes a 64-bit division.  Loads go first: their latency passes behind the
// generator's products.  One group to a thread: with two and four, 262,144 x 512
// float16, repeated on the same tensors, took 99 and 95 us in place of 86 (float32 189
// and 191 for 184, bfloat16 with an addition 141 and 145 for 132), and 20,011 x 199
// bfloat16 with an addition 15.9 with four for 8.9.  Only many rows gathered from a
// large table of 16-bit values are faster with four (262,144 x 512 bfloat16 105 us for
// 118, float16 96 for 111); 100,003 x 199 of them are not (32 for 28).
template <class T, bool ADD, bool IDS>
__global__ __launch_bounds__(kBlock) void k_dropout(DropoutCall c) {
  const polyglot_dropout_args& a = c.a;
  const int64_t first = (int64_t)blockIdx.x * kBlock;
  const int64_t row0 = first / c.groups;
  const uint32_t col0 = (uint32_t)(first - row0 * c.groups);
  const uint32_t site = a.site + (a.site_dev ? *a.site_dev : 0u);
  const uint32_t place = col0 + threadIdx.x;
  const uint32_t q = rows_down(place, c);
  const int64_t r = row0 + q;
  const int col = (int)(place - q * c.groups) * 8;
  if (r >= a.rows) return;
  const int n = min(8, a.d - col);
  bool bad = false;
  int64_t from = r;
  if (IDS) {
    from = a.id_bytes == 8 ? static_cast<const int64_t*>(a.ids)[r]
                           : static_cast<const int32_t*>(a.ids)[r];
    bad = from < 0 || from >= a.table_rows;
    if (bad) {
      from = 0;
      atomicOr(c.flag, kFlagBadId);
    }
  }
  const T* x = static_cast<const T*>(a.x) + from * a.ld_x + col;
  const T* add = static_cast<const T*>(a.add) + r * a.ld_add + col;
  T* y = static_cast<T*>(a.y) + r * a.ld_y + col;
  Oct<T> xv, av;
  if (n == 8) {
    xv.load(x);
    if (ADD) av.load(add);
  }
  const uint64_t row = a.first_row + (uint64_t)r;
  const uint4 w = philox10(uint4{a.whole_rows ? 0xffffffffu : (uint32_t)col / 8, (uint32_t)row,
                                 (uint32_t)(row >> 32), site},
                           (uint32_t)a.seed, (uint32_t)(a.seed >> 32));
  uint32_t keep = keep_bits(w, c.threshold);
  if (a.whole_rows) keep = keep & 1u ? 0xffu : 0u;
  const float spoilt = IDS && bad ? __builtin_nanf("") : -0.f;  // (v + -0 is v, also for -0)
  if (n == 8) {
    float v[8];
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      v[j] = keep >> j & 1u ? settled(xv.get(j) * c.scale) : 0.f;
      if (ADD) v[j] += av.get(j);
      if (IDS) v[j] += spoilt;
    }
    Oct<T>::store(y, v);
  } else {
    for (int j = 0; j < n; ++j) {
      float v = keep >> j & 1u ? settled(Elem<T>::get(x[j]) * c.scale) : 0.f;
      if (ADD) v += Elem<T>::get(add[j]);
      if (IDS) v += spoilt;
      y[j] = Elem<T>::put(settled(v));
    }
  }
}

}  // namespace pg
