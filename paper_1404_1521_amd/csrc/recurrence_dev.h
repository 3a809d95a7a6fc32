// Gated linear recurrence over packed sequences, and its gradient.
#pragma once
#include "formats.h"
#include "operators.h"

namespace pg {

__device__ __forceinline__ int64_t seq_offset(const RecCall& c, int i) {
  if (!c.offsets) return (int64_t)i * (c.tokens / c.nseq);
  return c.offset_bytes == 8 ? static_cast<const int64_t*>(c.offsets)[i]
                             : static_cast<const int32_t*>(c.offsets)[i];
}

// What a gate does: the decay a, and for a gate before its sigmoid the products
// with 1 - a and with the sigmoid's slope a (1 - a).  With s = e^(-|gate| / 2),
// r = 1 / (1 + s^2) and q = s r, the larger one of a and 1 - a is r, the other s q,
// and the slope q^2: nothing is lost to a subtraction, and a product taken factor
// by factor keeps its digits where 1 - a alone is below the normal floats.  The
// hardware's base-2 exponential and reciprocal (one unit in the last place).
struct Decay {
  float a, q, u, w;
  __device__ __forceinline__ float rest(float v) const { return v * u * w; }
  __device__ __forceinline__ float slope(float v) const { return v * q * q; }
};
template <int FORM>
__device__ __forceinline__ Decay decay(float g) {
  if constexpr (FORM == POLYGLOT_GATE_RAW) return Decay{g, 1.f, 1.f, 1.f};
  const float s = __builtin_amdgcn_exp2f(-0.72134752044448170f * __builtin_fabsf(g));
  const float r = __builtin_amdgcn_rcpf(1.f + s * s), q = s * r;
  return g >= 0.f ? Decay{r, q, q, s} : Decay{s * q, q, r, 1.f};
}

// A thread per sequence and channel, a workgroup per sequence and a range of
// channels that holds whole groups.
template <class T, int FORM, bool GRAD>
__global__ __launch_bounds__(kBlock) void k_recurrence(RecCall c) {
  __shared__ float part[kBlock];
  const int width = c.group > 1 ? kBlock / c.group * c.group : kBlock;  // channels per workgroup
  const int s = blockIdx.x, t = threadIdx.x, ch = blockIdx.y * width + t;
  const bool live = t < width && ch < c.D;
  int64_t lo = seq_offset(c, s), hi = seq_offset(c, s + 1);
  if (lo < 0 || hi < lo || hi > c.tokens || (s == 0 && lo != 0) ||
      (s == c.nseq - 1 && hi != c.tokens)) {
    if (t == 0) atomicOr(c.flag, kFlagBadOffset);
    lo = min(max(lo, (int64_t)0), (int64_t)c.tokens);
    hi = min(max(hi, lo), (int64_t)c.tokens);
  }
  const int gate_col = ch / c.group;
  float state = live && c.init ? c.init[(size_t)s * c.D + ch] : 0.f;
  for (int64_t i = 0; i < hi - lo; ++i) {
    const int64_t n = c.down ? hi - 1 - i : lo + i;
    float dg = 0.f;
    if (live) {
      const Decay k = decay<FORM>(
          Elem<T>::get(static_cast<const T*>(c.gate)[n * c.ld_gate + gate_col]));
      if constexpr (GRAD) {
        const float lam = Elem<T>::get(static_cast<const T*>(c.dh)[n * c.ld_dh + ch]) + state;
        const int64_t before = c.down ? n - 1 : n + 1;
        float h = 0.f;
        if (i + 1 < hi - lo) h = Elem<T>::get(static_cast<const T*>(c.h)[before * c.ld_h + ch]);
        else if (c.h0) h = c.h0[(size_t)s * c.D + ch];
        if constexpr (FORM == POLYGLOT_GATE_SIGMOID) {
          const float x = Elem<T>::get(static_cast<const T*>(c.x)[n * c.ld_x + ch]);
          dg = k.slope(lam * (h - x));
        } else {
          dg = lam * h;
        }
        static_cast<T*>(c.out)[n * c.ld_out + ch] = Elem<T>::put(k.rest(lam));
        state = k.a * lam;
      } else {
        const float x = Elem<T>::get(static_cast<const T*>(c.x)[n * c.ld_x + ch]);
        state = k.a * state + k.rest(x);
        static_cast<T*>(c.out)[n * c.ld_out + ch] = Elem<T>::put(state);
      }
    }
    if constexpr (GRAD) {
      T* dgate = static_cast<T*>(c.dgate) + n * c.ld_dgate;
      if (c.group == 1) {
        if (live) dgate[ch] = Elem<T>::put(dg);
      } else {
        __syncthreads();
        part[t] = dg;
        __syncthreads();
        if (live && t % c.group == 0) {
          float sum = 0.f;
          for (int j = 0; j < c.group; ++j) sum += part[t + j];
          dgate[gate_col] = Elem<T>::put(sum);
        }
      }
    }
  }
  if (live && c.fin) c.fin[(size_t)s * c.D + ch] = state;
}

}  // namespace pg
