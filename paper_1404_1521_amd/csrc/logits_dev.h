// A vocabulary's scores made ready for a choice: penalties for repeated words,
// biases, a mask of allowed words; the choice and the row's log-sum-exp.
//
// A workgroup takes a part of a row, up to 8,192 words, into registers, counts
// the row's history in LDS, one counter for each of its words, and applies the
// rules on the way out: the scores are read once and written once.  The parts of
// a row are joined by the workgroup that finishes last, from words in memory that
// carry the launch's tag, in the order of the parts.
//
// Bound by memory for many rows: 256 rows of 1,000,000 bfloat16 with histories of up to
// 4,096 ids 239 us (4.3 TB/s of 1.03 GB; copying the scores takes 208); without
// histories, which every part of a row reads again, 194.  A few rows: a chain of
// dependent rounds, the part's loads, the counts, the join's counter and words: one row
// of 100,000 float32 7.2 us, 48 of 32,003 bfloat16 8.9 us.
#pragma once
#include <type_traits>

#include "formats.h"
#include "operators.h"

namespace pg {

constexpr uint32_t kLogitsSpinLimit = 1u << 22;  // a wait that only a library bug makes
// A counter of the words that a workgroup holds: its top bit says that the word is in
// the history, the others count its made part.  16 bits, two counters to a word of LDS,
// for histories of at most 32,767 ids; 32 bits for longer ones.
template <bool LONG>
struct Counters {
  static constexpr int kBits = LONG ? 32 : 16;
  static constexpr uint32_t kIn = 1u << (kBits - 1);
  static constexpr int words(int n) { return LONG ? n : n / 2; }
  static __device__ __forceinline__ void add(uint32_t* c, int i, bool made) {
    uint32_t* w = c + (LONG ? i : i >> 1);
    const int shift = LONG ? 0 : 16 * (i & 1);
    atomicOr(w, kIn << shift);
    if (made) atomicAdd(w, 1u << shift);
  }
  // The four from i on (i a multiple of four).
  static __device__ __forceinline__ void quad(const uint32_t* c, int i, uint32_t (&k)[4]) {
    if constexpr (LONG) {
      const uint4 q = *reinterpret_cast<const uint4*>(c + i);
      k[0] = q.x, k[1] = q.y, k[2] = q.z, k[3] = q.w;
    } else {
      const uint2 q = *reinterpret_cast<const uint2*>(c + i / 2);
      k[0] = q.x & 0xffffu, k[1] = q.x >> 16, k[2] = q.y & 0xffffu, k[3] = q.y >> 16;
    }
  }
};

struct RowRules {
  float rep, freq, pres;
};
// Products and sums are kept apart: a fused multiply-add would round other scores
// to equal, or equal ones apart.
__device__ __forceinline__ float ruled(float l, uint32_t seen, uint32_t in, const RowRules& k) {
  if (seen) l = l > 0.f ? __fdiv_rn(l, k.rep) : __fmul_rn(l, k.rep);
  const uint32_t n = seen & ~in;
  if (n) l = __fsub_rn(l, __fadd_rn(__fmul_rn(k.freq, (float)n), k.pres));
  return l;
}

__device__ __forceinline__ float exp_fast(float x) {
  return __builtin_amdgcn_exp2f(1.44269504088896341f * x);
}

// e^l over a base no smaller than any l of a sum, where an infinity may be: equal
// infinities count once, a base of -infinity has no terms.
__device__ __forceinline__ float exp_over(float l, float base) {
  if (l == base) return base == -__builtin_inff() ? 0.f : 1.f;
  return exp_fast(l - base);
}

// Reductions over a wave in a fixed order, with DPP moves (as wave_incl_scan); the
// result is in every lane.
template <class V, class Op>
__device__ __forceinline__ V wave_reduce(V v, V none, Op op) {
  const auto moved = [&](auto ctrl, auto rows) {
    return __builtin_bit_cast(
        V, __builtin_amdgcn_update_dpp(__builtin_bit_cast(int, none), __builtin_bit_cast(int, v),
                                       decltype(ctrl)::value, decltype(rows)::value, 0xf, false));
  };
  v = op(v, moved(std::integral_constant<int, 0x111>{}, std::integral_constant<int, 0xf>{}));
  v = op(v, moved(std::integral_constant<int, 0x112>{}, std::integral_constant<int, 0xf>{}));
  v = op(v, moved(std::integral_constant<int, 0x114>{}, std::integral_constant<int, 0xf>{}));
  v = op(v, moved(std::integral_constant<int, 0x118>{}, std::integral_constant<int, 0xf>{}));
  v = op(v, moved(std::integral_constant<int, 0x142>{}, std::integral_constant<int, 0xa>{}));
  v = op(v, moved(std::integral_constant<int, 0x143>{}, std::integral_constant<int, 0xc>{}));
  return __builtin_bit_cast(V, __builtin_amdgcn_readlane(__builtin_bit_cast(int, v), 63));
}

// LDS of the reductions.
struct LogitsLds {
  float m[kWavesPerBlock], s[kWavesPerBlock];
  int w[kWavesPerBlock];
  uint64_t arrived;
};

constexpr int kNoWord = 0x7fffffff;

// The workgroup's largest m; its lowest w and its sum of s.  Every thread gets them.
__device__ __forceinline__ float largest(float m, LogitsLds& l) {
  m = wave_reduce(m, -__builtin_inff(), [](float a, float b) { return fmaxf(a, b); });
  if ((threadIdx.x & (kWave - 1)) == 0) l.m[threadIdx.x / kWave] = m;
  __syncthreads();
  m = l.m[0];
#pragma unroll
  for (int i = 1; i < kWavesPerBlock; ++i) m = fmaxf(m, l.m[i]);
  return m;
}
__device__ __forceinline__ void lowest_and_sum(int& w, float& s, LogitsLds& l) {
  w = wave_reduce(w, kNoWord, [](int a, int b) { return min(a, b); });
  s = wave_reduce(s, 0.f, [](float a, float b) { return a + b; });
  if ((threadIdx.x & (kWave - 1)) == 0) l.w[threadIdx.x / kWave] = w, l.s[threadIdx.x / kWave] = s;
  __syncthreads();
  w = l.w[0];
  s = l.s[0];
#pragma unroll
  for (int i = 1; i < kWavesPerBlock; ++i) w = min(w, l.w[i]), s += l.s[i];
}

// A part's or a row's log-sum-exp of sum s over base m.
__device__ __forceinline__ float log_sum(float m, float s) {
  if (s != s) return s;
  return __builtin_isinf(m) ? m : m + 0.69314718055994531f * __builtin_amdgcn_logf(s);
}

__device__ __forceinline__ void publish_word(uint64_t* w, uint32_t v, uint32_t tag) {
  __hip_atomic_store(w, (uint64_t)tag << 32 | v, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
}
// A word that has been or is being published with this tag.
__device__ __forceinline__ uint32_t await_word(const uint64_t* w, uint32_t tag, uint32_t* flag) {
  for (uint32_t spins = 0;; ++spins) {
    const uint64_t x = __hip_atomic_load(w, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
    if ((uint32_t)(x >> 32) == tag) return (uint32_t)x;
    if (spins > kLogitsSpinLimit) {
      atomicOr(flag, kFlagInternal);
      return 0;
    }
    __builtin_amdgcn_s_sleep(1);
  }
}

// The quad at place v of a row of V: the load stays inside the row, and what lies
// past its end is shifted out (whole: nothing does).  V < 4: word by word.
template <class T>
__device__ __forceinline__ Quad<T> row_quad(const T* row, int v, int V, bool whole) {
  if (V < 4) return load_quad<T, false>(row + min(v, V), max(0, min(4, V - v)));
  Quad<T> q = load_quad<T, true>(row + (whole ? v : min(v, V - 4)), 4);
  if (!whole) {
    const int off = max(0, min(3, v - (V - 4)));  // elements before v
    if constexpr (sizeof(T) == 2) {
      const uint64_t w = ((uint64_t)q.raw.y << 32 | q.raw.x) >> (16 * off);
      q.raw = u2_any{(uint32_t)w, (uint32_t)(w >> 32)};
    } else {
      if (off & 1) q.raw = f4{q.raw[1], q.raw[2], q.raw[3], 0.f};
      if (off & 2) q.raw = f4{q.raw[2], q.raw[3], 0.f, 0.f};
    }
  }
  return q;
}

// E words per thread, in quads 4 * 256 words apart.
template <class T, int E, bool LONG>
__global__ __launch_bounds__(kBlock) void k_logits(LogitsCall c) {
  constexpr int Q = E / 4, kWords = E * kBlock;  // the part's words
  using Count = Counters<LONG>;
  __shared__ __align__(16) uint32_t seen[Count::words(kWords)];
  __shared__ uint32_t allowed[kWords / 32];
  __shared__ LogitsLds lds;
  const polyglot_logits_args& a = c.a;
  const int t = threadIdx.x;
  const int r = blockIdx.x / c.tiles, tile = blockIdx.x - r * c.tiles;
  const int v0 = tile * (E * kBlock) + 4 * t;      // the thread's first word
  const bool whole = (tile + 1) * (E * kBlock) <= a.V;  // no quad of the part passes the row's end
  const T* in = static_cast<const T*>(a.logits) + (int64_t)r * a.ld_logits;
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
  // the part's scores, its part of the mask and the first of the history in flight: the
  // history up to what there is room for, what its length leaves out is skipped later
  constexpr int kAhead = 8;
  const int32_t* hist = a.history ? a.history + (int64_t)r * a.ld_history : nullptr;
  int id[kAhead];
  if (hist) {
#pragma unroll
    for (int j = 0; j < kAhead; ++j)
      id[j] = t + j * kBlock < a.history_cap ? hist[t + j * kBlock] : -1;
  }
  Quad<T> x[Q];
#pragma unroll
  for (int g = 0; g < Q; ++g) x[g] = row_quad<T>(in, v0 + g * 4 * kBlock, a.V, whole);
  constexpr int kMaskWords = kWords / 32;
  static_assert(kMaskWords <= kBlock, "a word of the mask for each thread");
  uint32_t bits = 0;
  if (mask && t < kMaskWords) bits = mask[min(tile * kMaskWords + t, (a.V - 1) >> 5)];
  uint32_t tag = 0;
  if (c.head && t == 0)  // the row's tag moves on once all its parts are in
    tag = (uint32_t)(__hip_atomic_load(c.head + r * kHeadLine, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT) >> 32);
  const RowRules rules{a.repetition ? a.repetition[r] : 1.f, a.frequency ? a.frequency[r] : 0.f,
                       a.presence ? a.presence[r] : 0.f};
  int len = 0, prompt = 0;
  if (a.history) {
    len = a.lengths ? min(max(a.lengths[r], 0), a.history_cap) : a.history_cap;
    prompt = a.prompt ? min(max(a.prompt[r], 0), a.history_cap) : 0;
  }
  if (len > 0) {
    uint4* const z = reinterpret_cast<uint4*>(seen);
    for (int i = t; i < Count::words(kWords) / 4; i += kBlock) z[i] = uint4{0u, 0u, 0u, 0u};
  }
  if (mask && t < kMaskWords) allowed[t] = bits;
  if (len > 0 || mask) __syncthreads();
  if (len > 0) {
    const int first = tile * kWords;
    for (int k0 = t;;) {
#pragma unroll
      for (int j = 0; j < kAhead; ++j) {
        const int k = k0 + j * kBlock;
        if (k >= len) continue;
        if (id[j] >= a.V) atomicOr(c.flag, kFlagBadId);
        else if (id[j] >= first && id[j] - first < kWords) Count::add(seen, id[j] - first, k >= prompt);
      }
      k0 += kAhead * kBlock;
      if (k0 - t >= len) break;
#pragma unroll
      for (int j = 0; j < kAhead; ++j) id[j] = k0 + j * kBlock < len ? hist[k0 + j * kBlock] : -1;
    }
    __syncthreads();
  }
  float l[E];
#pragma unroll
  for (int g = 0; g < Q; ++g) {
#pragma unroll
    for (int j = 0; j < 4; ++j) l[4 * g + j] = x[g].get(j);
    if (len > 0) {
      uint32_t k[4];
      Count::quad(seen, (g * kBlock + t) * 4, k);
      if (k[0] | k[1] | k[2] | k[3]) {
#pragma unroll
        for (int j = 0; j < 4; ++j) l[4 * g + j] = ruled(l[4 * g + j], k[j], Count::kIn, rules);
      }
    }
  }
  if (bias) {
    Quad<float> b[Q];
#pragma unroll
    for (int g = 0; g < Q; ++g) b[g] = row_quad<float>(bias, v0 + g * 4 * kBlock, a.V, whole);
#pragma unroll
    for (int i = 0; i < E; ++i) l[i] = __fadd_rn(l[i], b[i / 4].get(i & 3));
  }
  if (mask) {
#pragma unroll
    for (int g = 0; g < Q; ++g) {
      const int v = (g * kBlock + t) * 4;
      const uint32_t allow = allowed[v >> 5] >> (v & 31);
#pragma unroll
      for (int j = 0; j < 4; ++j)
        if (!(allow >> j & 1u)) l[4 * g + j] = -__builtin_inff();
    }
  }
  if (a.out) {
    T* out = static_cast<T*>(a.out) + (int64_t)r * a.ld_out;
#pragma unroll
    for (int g = 0; g < Q; ++g) {
      const int v = v0 + g * 4 * kBlock;
      const float o[4] = {l[4 * g], l[4 * g + 1], l[4 * g + 2], l[4 * g + 3]};
      if (whole || v + 4 <= a.V) store_quad<T, true>(out + v, o, 4);
      else store_quad<T, false>(out + min(v, a.V), o, a.V - v);
    }
  }
  if (!c.head) return;
  if (!whole) {
#pragma unroll
    for (int i = 0; i < E; ++i)
      if (v0 + (i / 4) * 4 * kBlock + (i & 3) >= a.V) l[i] = -__builtin_inff();
  }

  // the part's largest score, its first word, and the sum over that score
  float own = -__builtin_inff();
#pragma unroll
  for (int i = 0; i < E; ++i) own = fmaxf(own, l[i]);
  const float m = largest(own, lds);
  int w = kNoWord;
  if (own == m && m > -__builtin_inff()) {
#pragma unroll
    for (int i = E - 1; i >= 0; --i)
      if (l[i] == m) w = v0 + (i / 4) * 4 * kBlock + (i & 3);
  }
  float s = 0.f;
  if (a.lse) {
    if (__builtin_isinf(m)) {
      for (int i = 0; i < E; ++i) s += exp_over(l[i], m);
    } else {
#pragma unroll
      for (int i = 0; i < E; ++i) s += exp_fast(l[i] - m);
    }
  }
  lowest_and_sum(w, s, lds);
  if (c.tiles == 1) {
    if (t == 0) {
      if (a.token) a.token[r] = w == kNoWord ? -1 : w;
      if (a.lse) a.lse[r] = log_sum(m, s);
    }
    return;
  }
  uint64_t* words = c.words + (int64_t)r * c.stride * 3;
  if (t == 0) {
    publish_word(words + tile * 3, __float_as_uint(m), tag);
    publish_word(words + tile * 3 + 1, (uint32_t)w, tag);
    publish_word(words + tile * 3 + 2, __float_as_uint(s), tag);
    lds.arrived = __hip_atomic_fetch_add(c.head + r * kHeadLine, (uint64_t)1, __ATOMIC_RELAXED,
                                         __HIP_MEMORY_SCOPE_AGENT);
  }
  __syncthreads();
  if ((uint32_t)lds.arrived != (uint32_t)c.tiles - 1) {
    // More parts than the row has: another call, which the program lets overlap with
    // this one, counted in some of its own.
    if (t == 0 && (uint32_t)lds.arrived >= (uint32_t)c.tiles) atomicOr(c.flag, kFlagInternal);
    return;
  }

  // the last part joins them, in their order
  tag = (uint32_t)(lds.arrived >> 32);
  float top = -__builtin_inff();
  for (int j = t; j < c.tiles; j += kBlock)
    top = fmaxf(top, __uint_as_float(await_word(words + j * 3, tag, c.flag)));
  top = largest(top, lds);
  w = kNoWord;
  s = 0.f;
  for (int j = t; j < c.tiles; j += kBlock) {
    const float pm = __uint_as_float(await_word(words + j * 3, tag, c.flag));
    if (pm == top) w = min(w, (int)await_word(words + j * 3 + 1, tag, c.flag));
    s += __uint_as_float(await_word(words + j * 3 + 2, tag, c.flag)) * exp_over(pm, top);
  }
  lowest_and_sum(w, s, lds);
  if (t == 0) {
    if (a.token) a.token[r] = w == kNoWord ? -1 : w;
    if (a.lse) a.lse[r] = log_sum(top, s);
    const uint32_t next = tag + 1 ? tag + 1 : 1u;
    __hip_atomic_store(c.head + r * kHeadLine, (uint64_t)next << 32, __ATOMIC_RELAXED,
                       __HIP_MEMORY_SCOPE_AGENT);
  }
}

}  // namespace pg
