// Selective state space scan over packed sequences, and its gradient:
//   h_t[c][n] = a h_{t-1}[c][n] + D_t[c] x_t[c] B_t[n],   a = e^(D_t[c] A[c][n])
//   v_t[c] = sum_n C_t[n] h_t[c][n] + skip[c] x_t[c],     y = v or v z sigmoid(z)
//
// A wave holds all states of a few channels: LN lanes of four states each for a channel,
// two channels to a lane.  A state costs an exponential (twice an operation's time) and four
// operations a token; what a token brings for a channel (its step D, D x) or a state (B, C)
// comes from LDS, where the workgroup has put a tile of 16 tokens, converted once.  The sum
// over the states goes over LN lanes by DPP moves.
//
// The tokens are cut into ranges, a workgroup for each range and block of channels.  A
// first launch takes every range that a sequence runs out of from the sequence's start in
// it, or from nothing, to the state at its end, with the sum of its steps: the range's
// whole decay is e^(A sum D).  The second takes those before it in and goes through
// its own tokens.
//
// What bounds it are vector instructions: an operation takes a wave 4 cycles, the exponential
// 8, a state and token 20 in the first launch and 24 in the second.  At 32,768 x 2,048
// bfloat16 with 16 states and a gate that is 137 and 164 us of the 212 and 320 measured; the
// bytes are 103.  The rest is what a token and channel take by themselves: softplus, the
// gate's sigmoid, conversions, LDS, the sum over lanes.  Every state has a decay of its own, so
// that nothing here is a matrix product.
#pragma once
#include "places_dev.h"

namespace pg {

constexpr float kLog2e = 1.44269504088896341f, kLn2 = 0.69314718055994531f;
constexpr int kSelTile = kSelectiveTile;  // tokens of a tile, and between two marks

__device__ __forceinline__ float exp2_fast(float x) { return __builtin_amdgcn_exp2f(x); }

// e^-|x|: the product with log2 e and what its rounding lost.  (From 2^-150 on it is zero
// for all that follows; |x| stays finite there.)
__device__ __forceinline__ float exp_neg(float x) {
  const float m = __builtin_fminf(__builtin_fabsf(x), 104.f);
  const float t = m * -kLog2e;
  const float r = __fmaf_rn(m, -kLog2e, -t);
  const float e = exp2_fast(t);
  return __fmaf_rn(e, r * kLn2, e);
}

// log(1 + e^v) = max(v, 0) + log(1 + e), e = e^-|v|, and log(1 + e) = 2 atanh(e / (2 + e));
// the argument is at most 1/3, and the Maclaurin series' first term left out, s^17 / 17, is
// below 2^-29 of s.  (max(v, 0) by a comparison: -infinity gives zero, NaN stays.)
__device__ __forceinline__ float softplus(float v, float e) {
  const float s = e * __builtin_amdgcn_rcpf(2.f + e), q = s * s;
  float p = 2.f / 15.f;
  p = __fmaf_rn(p, q, 2.f / 13.f);
  p = __fmaf_rn(p, q, 2.f / 11.f);
  p = __fmaf_rn(p, q, 2.f / 9.f);
  p = __fmaf_rn(p, q, 2.f / 7.f);
  p = __fmaf_rn(p, q, 2.f / 5.f);
  p = __fmaf_rn(p, q, 2.f / 3.f);
  const float l = __fmaf_rn(s * q, p, s + s);
  return l + (v < 0.f ? 0.f : v);
}
__device__ __forceinline__ float softplus(float v) { return softplus(v, exp_neg(v)); }
__device__ __forceinline__ float sigmoid(float v, float e) {  // with that e
  const float r = __builtin_amdgcn_rcpf(1.f + e);
  return v >= 0.f ? r : e * r;
}
__device__ __forceinline__ float sigmoid(float v) { return sigmoid(v, exp_neg(v)); }

// A value of another lane of the row of 16 (DPP).
template <int CTRL>
__device__ __forceinline__ float lane_moved(float v) {
  return __int_as_float(__builtin_amdgcn_update_dpp(0, __float_as_int(v), CTRL, 0xf, 0xf, true));
}
// A value that is computed at this place.  The compiler otherwise moves a sum to where it is
// read: the last step of a sum over lanes into the branch that stores it, where it takes an
// instruction more, a gradient's sum behind the loop, with all its terms in registers.
__device__ __forceinline__ void here(float& v) { asm volatile("" : "+v"(v)); }
// The sum over the LN lanes of a channel, in all of them: neighbours, pairs, the half row
// mirrored, the row mirrored.
template <int LN>
__device__ __forceinline__ float sum_states(float v) {
  if constexpr (LN > 1) v += lane_moved<0xb1>(v);
  if constexpr (LN > 2) v += lane_moved<0x4e>(v);
  if constexpr (LN > 4) v += lane_moved<0x141>(v);
  if constexpr (LN > 8) v += lane_moved<0x140>(v);
  here(v);
  return v;
}

// The kernels' arguments, one block.  They are more than the scalar registers hold: `again`
// hides where the block lies, so that a phase of a tile loads those it needs from the scalar
// cache.  (Kept all the way they went to lanes of vector registers and came back one vector
// instruction each, a third of a tile's staging.)
struct SelArgs {
  SelCall c;
  SelPlan p;
};
typedef const __attribute__((address_space(4))) SelArgs* SelArgsPtr;
__device__ __forceinline__ SelArgsPtr sel_args() {
  return (SelArgsPtr)__builtin_amdgcn_kernarg_segment_ptr();
}
__device__ __forceinline__ const SelArgs& again(SelArgsPtr p) {
  asm volatile("" : "+s"(p));
  return *(const SelArgs*)p;
}

// Lanes, channels and places of a workgroup with LN lanes to a channel.
template <int LN>
struct SelShape {
  static constexpr int W = sel_waves(LN), THREADS = W * kWave;
  static constexpr int RC = 2;             // channels of a lane
  static constexpr int CL = kWave / LN;    // lanes of a state
  static constexpr int CW = CL * RC;       // channels of a wave
  static constexpr int CB = CW * W;        // ... of a workgroup
  static constexpr int NP = 4 * LN;        // states, with the empty places
  static constexpr int QUADS = CB / 4;     // of a token's row
  static constexpr int EACH = (kSelTile * QUADS + THREADS - 1) / THREADS;  // of a thread
  static constexpr int STEP = THREADS / QUADS;  // tokens between two of a thread's
  static constexpr int STATES = (2 * kSelTile * LN + THREADS - 1) / THREADS;  // quads of B and C
  static_assert(CB == sel_channels(LN) && THREADS % QUADS == 0, "a thread keeps its channels");
};

// What a workgroup, a thread and a lane work on.
template <int LN>
struct SelPlace {
  using S = SelShape<LN>;
  int head, c0, nc;  // the head, the workgroup's first channel, its channels
  int qn, q0, k0;    // a thread's quad of channels: how many are there, the first; its first token
  int lane_c, nl;    // a lane's channels (of the workgroup) and states
  uint32_t rate;     // the byte offset of the lane's states in a row of A, or of a sequence
  __device__ __forceinline__ SelPlace(const SelCall& c, const SelPlan& p, int block) {
    const int t = threadIdx.x, Dg = c.D / c.groups;
    head = block / p.blocks;
    const int b = block - head * p.blocks;
    c0 = head * Dg + b * S::CB;
    nc = min(S::CB, Dg - b * S::CB);
    const int quad = t % S::QUADS;
    k0 = t / S::QUADS;
    qn = max(0, min(4, nc - 4 * quad));
    q0 = qn ? c0 + 4 * quad : c0;
    const int lane = t & (kWave - 1);
    nl = lane % LN;
    lane_c = t / kWave * S::CW + lane / LN * S::RC;
    rate = ((uint32_t)(c0 + lane_c) * c.N + 4 * nl) * 4;
  }
  __device__ __forceinline__ bool has(int r) const { return lane_c + r < nc; }
};

// The sum of n values `ld` apart, by a workgroup for kSumOutputs sums side by side: each
// thread takes every sixteenth value, and the sixteen sums are added in their order.  The
// first kSumOutputs threads have the results.
constexpr int kSumOutputs = 16;
__device__ __forceinline__ float sum_parts(const float* from, int64_t ld, int n, bool there) {
  constexpr int kSlices = kBlock / kSumOutputs;
  __shared__ float part[kBlock];
  float v = 0.f;
  if (there) {
#pragma unroll 8
    for (int i = threadIdx.x / kSumOutputs; i < n; i += kSlices) v += from[i * ld];
  }
  part[threadIdx.x] = v;
  __syncthreads();
  v = 0.f;
  if (threadIdx.x < kSumOutputs) {
#pragma unroll
    for (int i = 0; i < kSlices; ++i) v += part[i * kSumOutputs + threadIdx.x];
  }
  return v;
}

template <class T>
__device__ __forceinline__ Quad<T> some_quad(const T* p, int n) {
  return n == 4 ? load_quad<T, true>(p, 4) : load_quad<T, false>(p, n);
}
template <class T>
__device__ __forceinline__ void put_quad(T* p, const float (&v)[4], int n) {
  if (n == 4) store_quad<T, true>(p, v, 4);
  else store_quad<T, false>(p, v, n);
}
template <class T>
__device__ __forceinline__ float load_one(const T* p) { return Elem<T>::get(*p); }
// Four of a channel's values from q0 on (none there: zero).
__device__ __forceinline__ void load_four(const float* p, int q0, int qn, float (&v)[4]) {
#pragma unroll
  for (int j = 0; j < 4; ++j) v[j] = 0.f;
  if (!p || qn == 0) return;
  const Quad<float> q = some_quad(p + q0, qn);
#pragma unroll
  for (int j = 0; j < 4; ++j) v[j] = q.get(j);
}

// A thread's place in a tile of a tensor: an offset of 32 bits (rows are less than 2^25
// elements apart) behind the tile's row, which is the same for the whole wave.
struct RowSpot {
  uint32_t off;
  template <class T>
  static __device__ __forceinline__ RowSpot of(const T*, int64_t ld, int k0, int q0) {
    return RowSpot{((uint32_t)k0 * (uint32_t)ld + (uint32_t)q0) * (uint32_t)sizeof(T)};
  }
  template <class T>
  __device__ __forceinline__ T* at(T* base, int64_t ld, int64_t row) const {
    return reinterpret_cast<T*>(reinterpret_cast<uintptr_t>(base + row * ld) + off);
  }
};

// A lane's four states of channel r, in A or in a sequence's states (row: the same for the
// whole wave); none past N: zero, and back.
template <int LN>
__device__ __forceinline__ void load_states(const float* row, const SelPlace<LN>& w, int r, int N,
                                            float (&h)[4]) {
#pragma unroll
  for (int j = 0; j < 4; ++j) h[j] = 0.f;
  const int n = N - 4 * w.nl;
  if (!row || !w.has(r) || n <= 0) return;
  const float* p = reinterpret_cast<const float*>(reinterpret_cast<uintptr_t>(row + r * N) + w.rate);
  const Quad<float> q = some_quad(p, min(n, 4));
#pragma unroll
  for (int j = 0; j < 4; ++j) h[j] = q.get(j);
}
template <int LN>
__device__ __forceinline__ void store_states(float* row, const SelPlace<LN>& w, int r, int N,
                                             const float (&h)[4]) {
  const int n = N - 4 * w.nl;
  if (!row || !w.has(r) || n <= 0) return;
  float* p = reinterpret_cast<float*>(reinterpret_cast<uintptr_t>(row + r * N) + w.rate);
  if (n >= 4) {
    *reinterpret_cast<f4_any*>(p) = f4_any{h[0], h[1], h[2], h[3]};
  } else {
#pragma unroll
    for (int j = 0; j < 3; ++j)
      if (j < n) p[j] = h[j];
  }
}
// The row of sequence i in [nseq][D][N].
template <class F>
__device__ __forceinline__ F* state_row(F* base, int i, const SelCall& c) {
  return base ? base + (int64_t)i * c.D * c.N : nullptr;
}

template <int LN>
__device__ __forceinline__ void load_rates(const SelCall& c, const SelPlace<LN>& w, float (&A)[2][4]) {
#pragma unroll
  for (int r = 0; r < 2; ++r) {
    load_states(c.A, w, r, c.N, A[r]);
#pragma unroll
    for (int k = 0; k < 4; ++k) A[r][k] *= kLog2e;
  }
}

// A tile's quads of a tensor on their way to a thread.  whole: all of them are there.
template <class T, class S>
struct QuadTile {
  Quad<T> q[S::EACH];
  template <class W>
  __device__ __forceinline__ void load(const void* base, int64_t ld, RowSpot spot, int t0, int count, bool whole,
                                       const W& w) {
    const T* p = static_cast<const T*>(base);
    if (whole) {
#pragma unroll
      for (int e = 0; e < S::EACH; ++e) q[e] = load_quad<T, true>(spot.at(p, ld, t0 + e * S::STEP), 4);
    } else {
#pragma unroll
      for (int e = 0; e < S::EACH; ++e) {
        q[e] = Quad<T>{};
        if (w.k0 + e * S::STEP < count && w.qn > 0) q[e] = some_quad(spot.at(p, ld, t0 + e * S::STEP), w.qn);
      }
    }
  }
};
// All quads of a tile are there: no thread is idle, no token or channel missing.
template <class S, class W>
__device__ __forceinline__ bool whole_tile(const W& w, int count) {
  return kSelTile * S::QUADS >= S::THREADS && count == kSelTile && w.nc == S::CB;
}

// A tile's rows of B and C (one of them null: of the other alone) on their way to LDS.
template <class T, int LN>
struct StateTile {
  using S = SelShape<LN>;
  Quad<T> q[S::STATES];
  __device__ __forceinline__ void load(const void* B, int64_t ld_B, const void* C, int64_t ld_C, int t0, int count,
                                       int head, int N) {
#pragma unroll
    for (int e = 0; e < S::STATES; ++e) {
      const int i = threadIdx.x + e * S::THREADS, k = i / LN % kSelTile, n0 = 4 * (i % LN);
      const bool second = i >= kSelTile * LN;
      const T* base = static_cast<const T*>(second ? C : B);
      q[e] = Quad<T>{};
      const int n = min(4, N - n0);
      if (base && i < 2 * kSelTile * LN && k < count && n > 0)
        q[e] = some_quad(base + (t0 + (int64_t)k) * (second ? ld_C : ld_B) + (int64_t)head * N + n0, n);
    }
  }
  __device__ __forceinline__ void put(float* B, float* C) const {
#pragma unroll
    for (int e = 0; e < S::STATES; ++e) {
      const int i = threadIdx.x + e * S::THREADS, at = i % (kSelTile * LN) * 4;
      if (i >= 2 * kSelTile * LN) continue;
      st4((i >= kSelTile * LN ? C : B) + at, f4{q[e].get(0), q[e].get(1), q[e].get(2), q[e].get(3)});
    }
  }
};

// The place of a thread's quad in a tile's [tokens][channels]; -1 for a thread without one.
template <class S>
__device__ __forceinline__ int quad_place(int e) {
  const int i = threadIdx.x + e * S::THREADS;
  return kSelTile * S::QUADS >= S::THREADS || i < kSelTile * S::QUADS ? i * 4 : -1;
}
// A thread's steps of a tile: what comes in, its bias, softplus; none where no token or
// channel is.  slope: receives the softplus' slopes.
template <class T, int LN, bool SLOPE = false>
__device__ __forceinline__ void tile_steps(const QuadTile<T, SelShape<LN>>& raw, const float (&bias)[4],
                                           bool soft, const SelPlace<LN>& w, int count, bool whole,
                                           float (&d)[SelShape<LN>::EACH][4], float* slope = nullptr) {
  using S = SelShape<LN>;
#pragma unroll
  for (int e = 0; e < S::EACH; ++e)
#pragma unroll
    for (int j = 0; j < 4; ++j) d[e][j] = raw.q[e].get(j) + bias[j];
  if (soft) {
#pragma unroll
    for (int e = 0; e < S::EACH; ++e) {
      f4 of;
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        const float x = exp_neg(d[e][j]);
        if (SLOPE) of[j] = sigmoid(d[e][j], x);
        d[e][j] = softplus(d[e][j], x);
      }
      if (SLOPE && quad_place<S>(e) >= 0) st4(slope + quad_place<S>(e), of);
    }
  }
  if (!whole) {
#pragma unroll
    for (int e = 0; e < S::EACH; ++e)
#pragma unroll
      for (int j = 0; j < 4; ++j)
        if (w.k0 + e * S::STEP >= count || j >= w.qn) d[e][j] = 0.f;
  }
}

// Takes `many` ranges (or groups of them) in, the last of them `at`, each by its whole decay and
// what it adds, four of them asked for at a time.  fresh: nothing comes into the first.
template <int LN>
__device__ __forceinline__ void take_in(const float* sums, const float* states, int at, int many, int dir, bool fresh,
                                        const SelCall& c, const SelPlace<LN>& w, const float (&A)[2][4],
                                        float (&h)[2][4]) {
  using S = SelShape<LN>;
  constexpr int BATCH = 4;
  const int own = w.has(0) ? w.lane_c : 0, two = w.has(1) ? 1 : 0;
  for (int m = many - 1; m >= 0; m -= BATCH) {
    float d[BATCH][2];
    f4 s[BATCH][2];
#pragma unroll
    for (int b = 0; b < BATCH; ++b) {
      const int j = at - dir * max(m - b, 0);
#pragma unroll
      for (int r = 0; r < 2; ++r) {
        const int64_t row = (int64_t)j * c.D + w.c0 + own + r * two;
        d[b][r] = sums[row];
        s[b][r] = ld4(states + row * S::NP + 4 * w.nl);
      }
    }
#pragma unroll
    for (int b = 0; b < BATCH; ++b) {
      if (m - b < 0) continue;
      const bool alone = fresh && m - b == many - 1;
#pragma unroll
      for (int r = 0; r < 2; ++r)
#pragma unroll
        for (int k = 0; k < 4; ++k)
          h[r][k] = alone ? s[b][r][k] : __fmaf_rn(exp2_fast(d[b][r] * A[r][k]), h[r][k], s[b][r][k]);
    }
  }
}
// How many from `at` on, against dir, up to and with the first that does not pass its own
// carry on, at most `most`; found: there is one.  By a whole wave.
__device__ __forceinline__ int open_run(const uint32_t* info, int at, int dir, int most, bool& found) {
  for (int many = 0; many < most; many += kWave) {
    const int i = many + lane_id();
    const uint64_t end = __ballot(i < most && info[at - dir * min(i, most - 1)] != kSelOpen);
    if (end) {
      found = true;
      return many + __builtin_ctzll(end) + 1;
    }
  }
  found = false;
  return most;
}
// Whether kSelNear ranges or more are open one after the other across the place behind `end`:
// those up to and with it, and those that follow.  By a whole wave, half of it for each.
__device__ __forceinline__ bool open_across(const uint32_t* info, int end, int dir, int ranges) {
  static_assert(kSelNear == kWave / 2, "a lane for each");
  const int l = lane_id(), i = l < kSelNear ? end - dir * l : end + dir * (l - kSelNear + 1);
  const uint64_t closed = __ballot(i < 0 || i >= ranges || info[i] != kSelOpen);
  const int before = __builtin_ctzll(closed | 1ull << kSelNear);
  const int behind = __builtin_ctzll(closed >> kSelNear | 1ull << kSelNear);
  return before + behind >= kSelNear;
}
// The carry into a range from those before it (dir -1: the gradient's, from those after it):
// since the last that starts afresh, each by itself where they are few, otherwise those of its
// group and the groups before that.
template <int LN>
__device__ __forceinline__ void carry_into(const SelCall& c, const SelPlan& p, int range, int dir,
                                           const SelPlace<LN>& w, const float (&A)[2][4],
                                           float (&h)[2][4]) {
#pragma unroll
  for (int r = 0; r < 2; ++r)
#pragma unroll
    for (int k = 0; k < 4; ++k) h[r][k] = 0.f;
  const int all = dir > 0 ? range : p.ranges - 1 - range;  // before it
  bool found;
  const int many = open_run(p.info, range - dir, dir, p.groups ? min(all, kSelNear) : all, found);
  if (found || many == all) {
    take_in<LN>(p.sums, p.states, range - dir, many, dir, true, c, w, A, h);
    return;
  }
  const int group = range / kSelGroup, place = range % kSelGroup;
  const int near = min(all, dir > 0 ? place : kSelGroup - 1 - place);  // (all of them open)
  bool any;
  const int far = open_run(p.group_info, group - dir, dir, dir > 0 ? group : p.groups - 1 - group, any);
  take_in<LN>(p.group_sums, p.group_states, group - dir, far, dir, true, c, w, A, h);
  take_in<LN>(p.sums, p.states, range - dir, near, dir, false, c, w, A, h);
}

// What groups of ranges pass on together: a thread for four states of a channel, a row of
// workgroups for a group.
template <int LN>
__global__ __launch_bounds__(kBlock) void k_selective_groups(SelCall c, SelPlan p, int dir) {
  constexpr int NP = SelShape<LN>::NP;
  const int blocks = (int)(((int64_t)c.D * LN + kBlock - 1) / kBlock), g = blockIdx.x / blocks;
  // Nothing reads it but behind kSelNear open ranges.
  if (!open_across(p.info, dir > 0 ? min((g + 1) * kSelGroup, p.ranges) - 1 : g * kSelGroup, dir, p.ranges)) return;
  const int64_t i = (int64_t)(blockIdx.x - g * blocks) * kBlock + threadIdx.x;
  if (i >= (int64_t)c.D * LN) return;
  const int ch = (int)(i / LN), n0 = (int)(i % LN) * 4;
  float A[4], h[4] = {0.f, 0.f, 0.f, 0.f}, sum = 0.f;
#pragma unroll
  for (int k = 0; k < 4; ++k) A[k] = n0 + k < c.N ? c.A[(int64_t)ch * c.N + n0 + k] * kLog2e : 0.f;
  const int from = g * kSelGroup, many = min(kSelGroup, p.ranges - from);
  float d[kSelGroup];
  f4 s[kSelGroup];
  uint32_t kind[kSelGroup];
#pragma unroll
  for (int m = 0; m < kSelGroup; ++m) {
    const int j = from + (dir > 0 ? min(m, many - 1) : max(many - 1 - m, 0));
    const int64_t row = (int64_t)j * c.D + ch;
    kind[m] = p.info[j];
    d[m] = p.sums[row];
    s[m] = ld4(p.states + row * NP + n0);
  }
  uint32_t all = kSelOpen;
#pragma unroll
  for (int m = 0; m < kSelGroup; ++m) {
    if (m >= many) continue;
    if (kind[m] != kSelOpen) all = kSelClosed, sum = 0.f;
    if (kind[m] != kSelNone) sum += d[m];
#pragma unroll
    for (int k = 0; k < 4; ++k)
      h[k] = kind[m] == kSelNone ? 0.f
             : kind[m] == kSelOpen ? __fmaf_rn(exp2_fast(d[m] * A[k]), h[k], s[m][k]) : s[m][k];
  }
  const int64_t row = (int64_t)g * c.D + ch;
  st4(p.group_states + row * NP + n0, f4{h[0], h[1], h[2], h[3]});
  if (n0 == 0) p.group_sums[row] = sum;
  if (n0 == 0 && ch == 0) p.group_info[g] = all;
}
template <int LN>
hipError_t selective_groups(const SelCall& c, const SelPlan& p, int dir, const Launch& L) {
  if (!p.groups || p.ranges <= 1) return hipSuccess;
  const int64_t blocks = ((int64_t)c.D * LN + kBlock - 1) / kBlock;
  return pg_launch(k_selective_groups<LN>, dim3((uint32_t)(p.groups * blocks)), dim3(kBlock), 0, L, c, p, dir);
}

// A workgroup's tile in LDS.
template <int LN>
struct alignas(16) SelLds {
  using S = SelShape<LN>;
  float step[kSelTile * S::CB], dx[kSelTile * S::CB];
  float B[kSelTile * S::NP], C[kSelTile * S::NP];
  TileMarks marks;
};

// What a range passes on, to the workspace.
template <int LN>
__device__ __forceinline__ void pass_on(const SelCall& c, const SelPlan& p, int range, const SelPlace<LN>& w,
                                        const float (&h)[2][4], const float (&sum)[2]) {
  using S = SelShape<LN>;
#pragma unroll
  for (int r = 0; r < 2; ++r) {
    if (!w.has(r)) continue;
    const int64_t at = (int64_t)range * c.D + w.c0 + w.lane_c + r;
    st4(p.states + at * S::NP + 4 * w.nl, f4{h[r][0], h[r][1], h[r][2], h[r][3]});
    if (w.nl == 0) p.sums[at] = sum[r];
  }
}

// ---------------------------------------------------------------- forward

// What a range passes on, and where the first launch takes it up: from the start of the
// sequence that runs out of the range, its number seq, or from the range's first token if
// that sequence began before it (seq -1).  By a whole wave.
struct RangeEnd {
  int at, seq;
  uint32_t kind;
};
__device__ __forceinline__ RangeEnd range_end(const Packed& s, int lo, int hi) {
  RangeEnd r{hi, -1, kSelNone};
  if (hi >= s.tokens) return r;
  const int i = first_place(s, hi);  // the first offset >= hi
  if (i <= s.nseq && place_of(s, i) == hi) return r;
  const int o = i > 0 ? min(place_of(s, i - 1), hi - 1) : 0;
  const bool starts = o >= lo && i > 0;
  r.at = starts ? o : lo;
  r.seq = starts ? i - 1 : -1;
  r.kind = starts || lo == 0 ? kSelClosed : kSelOpen;
  return r;
}
// The gradient's: up to the end of the sequence that runs into the range, if it ends in it.
__device__ __forceinline__ RangeEnd range_start(const Packed& s, int lo, int hi) {
  RangeEnd r{lo, -1, kSelNone};
  if (lo == 0 || lo >= hi) return r;
  const int i = first_place(s, lo);
  const int o = i <= s.nseq ? place_of(s, i) : hi;
  if (o == lo) return r;
  const bool ends = o <= hi && i > 0 && i <= s.nseq;
  r.at = max(lo, min(o, hi));
  r.seq = ends ? i - 1 : -1;
  r.kind = ends ? kSelClosed : kSelOpen;
  return r;
}

// The next tile is on its way while one is worked on.  A range costs here what it costs
// again below, without C, z and y: splitting time is what fills the chip (8 sequences of 2,048
// channels alone are 128 workgroups), and correcting outputs behind a single pass would take
// the same exponential and products of every state.  4,097 x 2,048, one sequence: 34 us.
template <class T, int LN>
__global__ __launch_bounds__(SelShape<LN>::THREADS) void k_selective_ends(SelArgs) {
  using S = SelShape<LN>;
  __shared__ SelLds<LN> s;
  const SelArgsPtr args = sel_args();
  const SelArgs& first = again(args);
  const int t = threadIdx.x;
  const int range = blockIdx.x / first.p.all_blocks, block = blockIdx.x % first.p.all_blocks;
  const SelPlace<LN> w(first.c, first.p, block);
  const int lo = first.p.share.first(range, kSelTile, first.c.seqs.tokens);
  const int hi = first.p.share.first(range + 1, kSelTile, first.c.seqs.tokens);
  const RangeEnd end = range_end(first.c.seqs, lo, hi);
  const int from = end.at, seq = end.seq;
  if (t == 0 && block == 0) first.p.info[range] = end.kind;
  if (end.kind == kSelNone) return;

  const RowSpot xs = RowSpot::of((const T*)nullptr, first.c.ld_x, w.k0, w.q0);
  const RowSpot ds = RowSpot::of((const T*)nullptr, first.c.ld_delta, w.k0, w.q0);
  QuadTile<T, S> xn, dn;  // the next tile's
  StateTile<T, LN> bn;
  const auto fetch = [&](int t0) {
    const SelCall& c = again(args).c;
    const int count = min(kSelTile, hi - t0);
    const bool whole = whole_tile<S>(w, count);
    dn.load(c.delta, c.ld_delta, ds, t0, count, whole, w);
    xn.load(c.x, c.ld_x, xs, t0, count, whole, w);
    bn.load(c.B, c.ld_B, nullptr, 0, t0, count, w.head, c.N);
  };
  fetch(from);
  float A[2][4], h[2][4], sum[2] = {0.f, 0.f}, bias[4];
  load_rates(first.c, w, A);
#pragma unroll
  for (int r = 0; r < 2; ++r)
    load_states(seq >= 0 ? state_row(first.c.h0, seq, first.c) : nullptr, w, r, first.c.N, h[r]);
  load_four(first.c.bias, w.q0, w.qn, bias);
  const bool soft = first.c.softplus;

  for (int t0 = from; t0 < hi; t0 += kSelTile) {
    const int count = min(kSelTile, hi - t0);
    __syncthreads();
    float d[S::EACH][4];
    tile_steps<T, LN>(dn, bias, soft, w, count, whole_tile<S>(w, count), d);
#pragma unroll
    for (int e = 0; e < S::EACH; ++e) {
      const int at = quad_place<S>(e);
      if (at < 0) continue;
      f4 u;
#pragma unroll
      for (int j = 0; j < 4; ++j) u[j] = d[e][j] * xn.q[e].get(j);
      st4(s.step + at, f4{d[e][0], d[e][1], d[e][2], d[e][3]});
      st4(s.dx + at, u);
    }
    bn.put(s.B, s.C);
    if (t0 + kSelTile < hi) fetch(t0 + kSelTile);
    __syncthreads();
#pragma unroll 4
    for (int k = 0; k < kSelTile; ++k) {  // (tokens past the range: no step, nothing added)
      const float2 d2 = *reinterpret_cast<const float2*>(s.step + k * S::CB + w.lane_c);
      const float2 u2 = *reinterpret_cast<const float2*>(s.dx + k * S::CB + w.lane_c);
      const f4 B = ld4(s.B + k * S::NP + 4 * w.nl);
      const float dd[2] = {d2.x, d2.y}, uu[2] = {u2.x, u2.y};
#pragma unroll
      for (int r = 0; r < 2; ++r) {
        sum[r] += dd[r];
#pragma unroll
        for (int j = 0; j < 4; ++j)
          h[r][j] = __fmaf_rn(exp2_fast(dd[r] * A[r][j]), h[r][j], uu[r] * B[j]);
      }
    }
  }
  const SelArgs& last = again(args);
  pass_on(last.c, last.p, range, w, h, sum);
}

// Four waves to a SIMD (128 registers).  Five left the tile's loads no room and spilled: both
// launches 5% longer at 32,768 x 2,048.  Tiles where no sequence starts or stops take a loop
// without a branch, four tokens unrolled (1% longer with two).  4,097 x 2,048: 63 us.
template <class T, int LN>
__global__ __launch_bounds__(SelShape<LN>::THREADS, 4) void k_selective(SelArgs) {
  using S = SelShape<LN>;
  __shared__ SelLds<LN> s;
  __shared__ __align__(16) float sy[kSelTile * S::CB];
  __shared__ int list[S::THREADS + 1];
  const SelArgsPtr args = sel_args();
  const SelArgs& first = again(args);
  const int t = threadIdx.x;
  const int range = blockIdx.x / first.p.all_blocks, block = blockIdx.x % first.p.all_blocks;
  const SelPlace<LN> w(first.c, first.p, block);
  const int lo = first.p.share.first(range, kSelTile, first.c.seqs.tokens);
  const int hi = first.p.share.first(range + 1, kSelTile, first.c.seqs.tokens);

  check_places(first.c.seqs, range, first.p.ranges, S::THREADS, first.c.last != nullptr, list, [&](int i) {
    const SelCall& c = again(args).c;
    for (int r = 0; r < 2; ++r) {
      float v[4];
      load_states(state_row(c.h0, i, c), w, r, c.N, v);
      store_states(state_row(c.last, i, c), w, r, c.N, v);
    }
  });
  if (lo >= hi) return;

  const T* none = nullptr;
  const RowSpot xs = RowSpot::of(none, first.c.ld_x, w.k0, w.q0), ds = RowSpot::of(none, first.c.ld_delta, w.k0, w.q0);
  const RowSpot zs = RowSpot::of(none, first.c.ld_z, w.k0, w.q0), ys = RowSpot::of(none, first.c.ld_y, w.k0, w.q0);
  const bool gated = first.c.z != nullptr, soft = first.c.softplus;
  QuadTile<T, S> xn, dn, zv;  // the next tile's, and this one's z
  StateTile<T, LN> bn;
  const auto fetch = [&](int t0) {
    const SelCall& c = again(args).c;
    const int count = min(kSelTile, hi - t0);
    const bool whole = whole_tile<S>(w, count);
    dn.load(c.delta, c.ld_delta, ds, t0, count, whole, w);
    xn.load(c.x, c.ld_x, xs, t0, count, whole, w);
    bn.load(c.B, c.ld_B, c.C, c.ld_C, t0, count, w.head, c.N);
  };
  fetch(lo);
  float A[2][4], h[2][4], bias[4], skip[4];
  load_rates(first.c, w, A);
  load_four(first.c.bias, w.q0, w.qn, bias);
  load_four(first.c.skip, w.q0, w.qn, skip);
  const bool skips = first.c.skip != nullptr;
  UpCursor cursor{};
  {
    const SelArgs& a = again(args);
    const int next = first_place(a.c.seqs, lo);
    if (t < kWave) cursor.read(a.c.seqs, next);
    // unless a sequence starts here
    if (lo > 0 && !(next <= a.c.seqs.nseq && place_of(a.c.seqs, next) == lo)) {
      carry_into<LN>(a.c, a.p, range, 1, w, A, h);
    } else {
#pragma unroll
      for (int r = 0; r < 2; ++r)
#pragma unroll
        for (int j = 0; j < 4; ++j) h[r][j] = 0.f;
    }
  }

  for (int t0 = lo; t0 < hi; t0 += kSelTile) {
    const int count = min(kSelTile, hi - t0);
    const bool whole = whole_tile<S>(w, count);
    const QuadTile<T, S> xv = xn;
    float d[S::EACH][4];
    tile_steps<T, LN>(dn, bias, soft, w, count, whole, d);
#pragma unroll
    for (int e = 0; e < S::EACH; ++e) {
      const int at = quad_place<S>(e);
      if (at < 0) continue;
      f4 u;
#pragma unroll
      for (int j = 0; j < 4; ++j) u[j] = d[e][j] * xv.q[e].get(j);
      st4(s.step + at, f4{d[e][0], d[e][1], d[e][2], d[e][3]});
      st4(s.dx + at, u);
    }
    bn.put(s.B, s.C);
    if (t < kWave) mark_tile(again(args).c.seqs, t0, t0 + count, cursor, s.marks);
    __syncthreads();
    const uint32_t starts = __builtin_amdgcn_readfirstlane(s.marks.starts);
    const uint32_t stops = __builtin_amdgcn_readfirstlane(s.marks.stops);
    const SelArgs& a = again(args);
    if (gated) zv.load(a.c.z, a.c.ld_z, zs, t0, count, whole, w);
    if (t0 + kSelTile < hi) fetch(t0 + kSelTile);
    if (a.c.marks) {
#pragma unroll
      for (int r = 0; r < 2; ++r) {
        if (!w.has(r) || 4 * w.nl >= a.c.N) continue;
        const int64_t at = (int64_t)(t0 / kSelTile) * a.c.D + w.c0 + w.lane_c + r;
        st4(a.c.marks + at * a.p.NM + 4 * w.nl, f4{h[r][0], h[r][1], h[r][2], h[r][3]});
      }
    }
    const auto token = [&](int k) {
      const float2 d2 = *reinterpret_cast<const float2*>(s.step + k * S::CB + w.lane_c);
      const float2 u2 = *reinterpret_cast<const float2*>(s.dx + k * S::CB + w.lane_c);
      const f4 B = ld4(s.B + k * S::NP + 4 * w.nl), C = ld4(s.C + k * S::NP + 4 * w.nl);
      const float dd[2] = {d2.x, d2.y}, uu[2] = {u2.x, u2.y};
      float out[2];
#pragma unroll
      for (int r = 0; r < 2; ++r) {
        float v = 0.f;
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          h[r][j] = __fmaf_rn(exp2_fast(dd[r] * A[r][j]), h[r][j], uu[r] * B[j]);
          v = __fmaf_rn(C[j], h[r][j], v);
        }
        out[r] = sum_states<LN>(v);
      }
      if (w.nl == 0) *reinterpret_cast<float2*>(sy + k * S::CB + w.lane_c) = float2{out[0], out[1]};
    };
    if ((starts | stops) == 0) {  // (tokens past the range have no step and add nothing)
#pragma unroll 4
      for (int k = 0; k < kSelTile; ++k) token(k);
    } else {
      for (int k = 0; k < count; ++k) {
        if (starts >> k & 1) {
          const float* row = state_row(a.c.h0, __builtin_amdgcn_readfirstlane(s.marks.start[k]), a.c);
#pragma unroll
          for (int r = 0; r < 2; ++r) load_states(row, w, r, a.c.N, h[r]);
        }
        token(k);
        if (stops >> k & 1) {
          float* row = state_row(a.c.last, __builtin_amdgcn_readfirstlane(s.marks.stop[k]), a.c);
#pragma unroll
          for (int r = 0; r < 2; ++r) store_states(row, w, r, a.c.N, h[r]);
        }
      }
    }
    __syncthreads();
    const SelCall& c = again(args).c;
#pragma unroll
    for (int e = 0; e < S::EACH; ++e) {
      const int at = quad_place<S>(e);
      if (at < 0 || (!whole && (w.k0 + e * S::STEP >= count || w.qn == 0))) continue;
      const f4 q = ld4(sy + at);
      float v[4] = {q[0], q[1], q[2], q[3]};
      if (skips) {
#pragma unroll
        for (int j = 0; j < 4; ++j) v[j] = __fmaf_rn(skip[j], xv.q[e].get(j), q[j]);
      }
      if (gated) {
#pragma unroll
        for (int j = 0; j < 4; ++j) v[j] *= zv.q[e].get(j) * sigmoid(zv.q[e].get(j));
      }
      put_quad(ys.at(static_cast<T*>(c.y), c.ld_y, t0 + e * S::STEP), v, w.qn);
    }
  }
}

// One token for each sequence: LN lanes of four states each for a channel of a row, a channel
// to each group of lanes, so that a workgroup's states are one contiguous piece.  Its bytes are
// the states, in and out: 64 x 2,048 with 16 states 7.7 us for 18 MB, 3.4 at a copy's rate;
// the rest is one round trip of loads and the launch.
template <class T, int LN>
__global__ __launch_bounds__(kBlock) void k_selective_step(SelCall c, int blocks) {
  constexpr int CB = kBlock / LN;  // channels of a workgroup
  const int nl = threadIdx.x % LN;
  const int64_t all = (int64_t)c.seqs.nseq * blocks;
  for (int64_t i = blockIdx.x; i < all; i += gridDim.x) {
    const int64_t row = i / blocks;
    const int ch = (int)(i - row * blocks) * CB + threadIdx.x / LN;
    const bool live = ch < c.D;
    const int own = live ? ch : 0, head = own / (c.D / c.groups), n = min(4, c.N - 4 * nl);
    const int64_t at = (row * c.D + own) * c.N + 4 * nl;
    const int64_t bc = (int64_t)head * c.N + 4 * nl;
    Quad<float> A{}, h{};
    Quad<T> B{}, C{};
    if (n > 0) {
      if (c.h0) h = some_quad(c.h0 + at, n);
      A = some_quad(c.A + (int64_t)own * c.N + 4 * nl, n);
      B = some_quad(static_cast<const T*>(c.B) + row * c.ld_B + bc, n);
      C = some_quad(static_cast<const T*>(c.C) + row * c.ld_C + bc, n);
    }
    const float x = load_one(static_cast<const T*>(c.x) + row * c.ld_x + own);
    const float z = c.z ? load_one(static_cast<const T*>(c.z) + row * c.ld_z + own) : 0.f;
    float d = load_one(static_cast<const T*>(c.delta) + row * c.ld_delta + own);
    if (c.bias) d += c.bias[own];
    if (c.softplus) d = softplus(d);
    const float u = d * x;
    float v = 0.f, out[4];
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      out[j] = __fmaf_rn(exp2_fast(d * (A.get(j) * kLog2e)), h.get(j), u * B.get(j));
      v = __fmaf_rn(C.get(j), out[j], v);
    }
    v = sum_states<LN>(v);
    if (!live) continue;
    if (c.last && n > 0) put_quad(c.last + at, out, n);
    if (nl == 0) {
      if (c.skip) v = __fmaf_rn(c.skip[own], x, v);
      if (c.z) v *= z * sigmoid(z);
      static_cast<T*>(c.y)[row * c.ld_y + own] = Elem<T>::put(settled(v));
    }
  }
}

}  // namespace pg
