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

// The quotient n / groups of a workgroup's places, n < groups + kDropPlaces.
constexpr int kDropPlaces = 1024;
__device__ __forceinline__ uint32_t rows_down(uint32_t n, const DropoutCall& c) {
  if (c.groups >= kDropPlaces) return n >= (uint32_t)c.groups ? 1u : 0u;
  return c.groups == 1 ? n : __umulhi(n, c.groups_inv);
}

// A workgroup takes U * 256 consecutive groups of eight columns, counted through
// all rows.  Loads go first: their latency passes behind the generator's products.
template <class T, bool ADD, bool IDS, int U>
__global__ __launch_bounds__(kBlock) void k_dropout(DropoutCall c) {
  const polyglot_dropout_args& a = c.a;
  const int64_t first = (int64_t)blockIdx.x * (kBlock * U);
  const int64_t row0 = first / c.groups;
  const uint32_t col0 = (uint32_t)(first - row0 * c.groups);
  const uint32_t site = a.site + (a.site_dev ? *a.site_dev : 0u);
  int64_t r[U];
  int col[U], n[U];
  bool bad[U];
  const T* x[U];
#pragma unroll
  for (int u = 0; u < U; ++u) {
    const uint32_t place = col0 + threadIdx.x + u * kBlock;
    const uint32_t q = rows_down(place, c);
    r[u] = row0 + q;
    col[u] = (int)(place - q * c.groups) * 8;
    n[u] = r[u] < a.rows ? min(8, a.d - col[u]) : 0;
    bad[u] = false;
    int64_t from = r[u];
    if (IDS && n[u] > 0) {
      from = a.id_bytes == 8 ? static_cast<const int64_t*>(a.ids)[r[u]]
                             : static_cast<const int32_t*>(a.ids)[r[u]];
      bad[u] = from < 0 || from >= a.table_rows;
      if (bad[u]) {
        from = 0;
        atomicOr(c.flag, kFlagBadId);
      }
    }
    x[u] = static_cast<const T*>(a.x) + from * a.ld_x + col[u];
  }
  Oct<T> xv[U], av[U];
#pragma unroll
  for (int u = 0; u < U; ++u)
    if (n[u] == 8) {
      xv[u].load(x[u]);
      if (ADD) av[u].load(static_cast<const T*>(a.add) + r[u] * a.ld_add + col[u]);
    }
#pragma unroll
  for (int u = 0; u < U; ++u) {
    const uint64_t row = a.first_row + (uint64_t)r[u];
    const uint4 w = philox10(uint4{a.whole_rows ? 0xffffffffu : (uint32_t)col[u] / 8, (uint32_t)row,
                                   (uint32_t)(row >> 32), site},
                             (uint32_t)a.seed, (uint32_t)(a.seed >> 32));
    uint32_t keep = keep_bits(w, c.threshold);
    if (a.whole_rows) keep = keep & 1u ? 0xffu : 0u;
    const float spoilt = IDS && bad[u] ? __builtin_nanf("") : 0.f;
    T* y = static_cast<T*>(a.y) + r[u] * a.ld_y + col[u];
    if (n[u] == 8) {
      float v[8];
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        v[j] = keep >> j & 1u ? settled(xv[u].get(j) * c.scale) : 0.f;
        if (ADD) v[j] += av[u].get(j);
        if (IDS) v[j] += spoilt;
      }
      Oct<T>::store(y, v);
    } else {
      const T* add = static_cast<const T*>(a.add) + r[u] * a.ld_add + col[u];
      for (int j = 0; j < n[u]; ++j) {
        float v = keep >> j & 1u ? settled(Elem<T>::get(x[u][j]) * c.scale) : 0.f;
        if (ADD) v += Elem<T>::get(add[j]);
        if (IDS) v += spoilt;
        y[j] = Elem<T>::put(settled(v));
      }
    }
  }
}

}  // namespace pg
