// A vocabulary's scores made ready for a choice: penalties for repeated words,
// biases, a mask of allowed words; the choice and the row's log-sum-exp.
#pragma once
#include "formats.h"
#include "operators.h"

namespace pg {

constexpr int kLogitsTile = 8192;          // words whose counts are in LDS at a time
constexpr uint32_t kSeenOnly = 0x80000000u;  // in the history; the low bits count its made part

// The score of word v of a row.  Products and sums are kept apart: a fused
// multiply-add would round other scores to equal, or equal ones apart.
struct RowRules {
  float rep, freq, pres;
};
__device__ __forceinline__ float ruled(float l, uint32_t seen, const RowRules& k) {
  if (seen) l = l > 0.f ? __fdiv_rn(l, k.rep) : __fmul_rn(l, k.rep);
  const uint32_t n = seen & ~kSeenOnly;
  if (n) l = __fsub_rn(l, __fadd_rn(__fmul_rn(k.freq, (float)n), k.pres));
  return l;
}

// One workgroup per row.
template <class T>
__global__ __launch_bounds__(kBlock) void k_logits(LogitsCall c) {
  __shared__ uint32_t seen[kLogitsTile];
  __shared__ float red_m[kBlock], red_s[kBlock];
  __shared__ int red_v[kBlock];
  const polyglot_logits_args& a = c.a;
  const int r = blockIdx.x, t = threadIdx.x;
  const T* in = static_cast<const T*>(a.logits) + (int64_t)r * a.ld_logits;
  T* out = a.out ? static_cast<T*>(a.out) + (int64_t)r * a.ld_out : nullptr;
  const RowRules rules{a.repetition ? a.repetition[r] : 1.f, a.frequency ? a.frequency[r] : 0.f,
                       a.presence ? a.presence[r] : 0.f};
  const int32_t* hist = a.history ? a.history + (int64_t)r * a.ld_history : nullptr;
  int len = 0, prompt = 0;
  if (hist) {
    len = a.lengths ? min(max(a.lengths[r], 0), a.history_cap) : a.history_cap;
    prompt = a.prompt ? min(max(a.prompt[r], 0), a.history_cap) : 0;
  }
  const float* bias = a.bias ? a.bias + (int64_t)r * a.ld_bias : nullptr;
  const uint32_t* mask = nullptr;
  if (a.mask) {
    int m = a.mask_rows ? a.mask_rows[r] : (a.masks == 1 ? 0 : r);
    if (m >= a.masks) {
      if (t == 0) atomicOr(c.flag, kFlagBadId);
      m = -1;
    }
    if (m >= 0) mask = a.mask + (int64_t)m * a.ld_mask;
  }
  float best = -__builtin_inff(), top = -__builtin_inff(), sum = 0.f;
  int word = -1;
  for (int v0 = 0; v0 < a.V; v0 += kLogitsTile) {
    const int n = min(kLogitsTile, a.V - v0);
    __syncthreads();
    for (int i = t; i < n; i += kBlock) seen[i] = 0;
    __syncthreads();
    for (int k = t; k < len; k += kBlock) {
      const int id = hist[k];
      if (id >= a.V) atomicOr(c.flag, kFlagBadId);
      const int i = id - v0;
      if (id >= v0 && i < n) {
        atomicOr(&seen[i], kSeenOnly);
        if (k >= prompt) atomicAdd(&seen[i], 1u);
      }
    }
    __syncthreads();
    for (int i = t; i < n; i += kBlock) {
      const int v = v0 + i;
      float l = ruled(Elem<T>::get(in[v]), seen[i], rules);
      if (bias) l = __fadd_rn(l, bias[v]);
      if (mask && !(mask[v >> 5] >> (v & 31) & 1u)) l = -__builtin_inff();
      if (out) out[v] = Elem<T>::put(l);
      if (l > best) best = l, word = v;
      if (l > top) {
        if (top != -__builtin_inff()) sum *= __expf(top - l);
        top = l;
      }
      if (l != l) sum = l;
      else if (l != -__builtin_inff()) sum += l == top ? 1.f : __expf(l - top);
    }
  }
  red_m[t] = best;
  red_v[t] = word;
  red_s[t] = sum;
  __syncthreads();
  if (t != 0) return;
  for (int i = 1; i < kBlock; ++i) {
    if (red_m[i] > best || (red_m[i] == best && red_v[i] >= 0 && red_v[i] < word)) {
      best = red_m[i];
      word = red_v[i];
    }
  }
  if (a.token) a.token[r] = word;
  if (a.lse) {
    float s = 0.f;
    for (int i = 0; i < kBlock; ++i)
      s += red_m[i] == best ? red_s[i] : red_s[i] * __expf(red_m[i] - best);
    // infinities have no finite share of the sum
    a.lse[r] = s != s ? s : (best == __builtin_inff() || s == 0.f) ? best : best + __logf(s);
  }
}

}  // namespace pg
