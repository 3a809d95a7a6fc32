// Selective state space scan over packed sequences, and its gradient:
//   h_t[c][n] = a h_{t-1}[c][n] + D_t[c] x_t[c] B_t[n],   a = e^(D_t[c] A[c][n])
//   v_t[c] = sum_n C_t[n] h_t[c][n] + skip[c] x_t[c],     y = v or v z sigmoid(z)
//
// A wave holds all states of a few channels: LN lanes of four states each for a channel,
// two channels to a lane.  A state costs an exponential (a quarter of the vector rate)
// and four operations a token; what a token brings for a channel (its step D, D x) or a
// state (B, C) comes from LDS, where the workgroup has put a tile of 16 tokens, converted
// once.  The sum over the states goes over LN lanes by DPP moves.
//
// The tokens are cut into ranges, a workgroup for each range and block of channels.  A
// first launch takes every range that a sequence runs out of from the sequence's start in
// it, or from nothing, to the state at its end, with the sum of its steps: the range's
// whole decay is e^(A sum D).  The second takes those before it in and goes through
// its own tokens.
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
// below 2^-29 of s.
__device__ __forceinline__ float softplus(float v) {
  const float e = exp_neg(v);
  const float s = e * __builtin_amdgcn_rcpf(2.f + e), q = s * s;
  float p = 2.f / 15.f;
  p = __fmaf_rn(p, q, 2.f / 13.f);
  p = __fmaf_rn(p, q, 2.f / 11.f);
  p = __fmaf_rn(p, q, 2.f / 9.f);
  p = __fmaf_rn(p, q, 2.f / 7.f);
  p = __fmaf_rn(p, q, 2.f / 5.f);
  p = __fmaf_rn(p, q, 2.f / 3.f);
  const float l = __fmaf_rn(s * q, p, s + s);
  return __fmaf_rn(v + __builtin_fabsf(v), 0.5f, l);  // (NaN stays)
}
__device__ __forceinline__ float sigmoid(float v) {
  const float e = exp_neg(v);
  const float r = __builtin_amdgcn_rcpf(1.f + e);
  return v >= 0.f ? r : e * r;
}

// A value of another lane of the row of 16 (DPP).
template <int CTRL>
__device__ __forceinline__ float lane_moved(float v) {
  return __int_as_float(__builtin_amdgcn_update_dpp(0, __float_as_int(v), CTRL, 0xf, 0xf, true));
}
// The sum over the LN lanes of a channel, in all of them: neighbours, pairs, the half row
// mirrored, the row mirrored.
template <int LN>
__device__ __forceinline__ float sum_states(float v) {
  if constexpr (LN > 1) v += lane_moved<0xb1>(v);
  if constexpr (LN > 2) v += lane_moved<0x4e>(v);
  if constexpr (LN > 4) v += lane_moved<0x141>(v);
  if constexpr (LN > 8) v += lane_moved<0x140>(v);
  return v;
}

// Lanes, channels and places of a workgroup with LN lanes to a channel.
template <int LN>
struct SelShape {
  static constexpr int RC = 2;                    // channels of a lane
  static constexpr int CL = kWave / LN;           // lanes of a state
  static constexpr int CW = CL * RC;              // channels of a wave
  static constexpr int CB = CW * kWavesPerBlock;  // ... of a workgroup
  static constexpr int NP = 4 * LN;               // states, with the empty places
  static constexpr int QUADS = CB / 4;            // of a token's row
  static constexpr int EACH = (kSelTile * QUADS + kBlock - 1) / kBlock;  // of a thread
  static constexpr int STEP = kBlock / QUADS;     // tokens between two of a thread's
  static_assert(kBlock % QUADS == 0, "a thread keeps its channels from token to token");
};

// What a workgroup works on.
template <int LN>
struct SelPlace {
  using S = SelShape<LN>;
  int head, c0, nc;  // the head, the workgroup's first channel, its channels
  int quad, qn, q0;  // a thread's quad of channels in a row, how many are there, the first
  int k0;            // the first of a tile's tokens that the thread brings in
  int lane_c, nl;    // a lane's channels (of the workgroup) and states
  __device__ __forceinline__ SelPlace(const SelCall& c, const SelPlan& p, int block) {
    const int t = threadIdx.x, Dg = c.D / c.groups;
    head = block / p.blocks;
    const int b = block - head * p.blocks;
    c0 = head * Dg + b * S::CB;
    nc = min(S::CB, Dg - b * S::CB);
    quad = t % S::QUADS;
    k0 = t / S::QUADS;
    qn = max(0, min(4, nc - 4 * quad));
    q0 = qn ? c0 + 4 * quad : c0;
    const int lane = t & (kWave - 1);
    nl = lane % LN;
    lane_c = t / kWave * S::CW + lane / LN * S::RC;
  }
};

template <class T>
__device__ __forceinline__ Quad<T> some_quad(const T* p, int n) {
  return n == 4 ? load_quad<T, true>(p, 4) : load_quad<T, false>(p, n);
}
template <class T>
__device__ __forceinline__ void put_quad(T* p, const float (&v)[4], int n) {
  if (n == 4) store_quad<T, true>(p, v, 4);
  else store_quad<T, false>(p, v, n);
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

template <class T>
__device__ __forceinline__ float load_one(const T* p) { return Elem<T>::get(*p); }

// The states' rows: a lane's four of channel c (none past N: zero), and back.
__device__ __forceinline__ void load_states(const float* row, int N, int nl, float (&h)[4]) {
#pragma unroll
  for (int j = 0; j < 4; ++j) h[j] = row && 4 * nl + j < N ? row[4 * nl + j] : 0.f;
}
__device__ __forceinline__ void store_states(float* row, int N, int nl, const float (&h)[4]) {
#pragma unroll
  for (int j = 0; j < 4; ++j)
    if (4 * nl + j < N) row[4 * nl + j] = h[j];
}

// A tile's quads of a tensor on their way to a thread.
template <class T, class S>
struct QuadTile {
  Quad<T> q[S::EACH];
  __device__ __forceinline__ void load(const T* base, int64_t ld, RowSpot spot, int t0, int count, int k0,
                                       int qn) {
#pragma unroll
    for (int e = 0; e < S::EACH; ++e) {
      q[e] = Quad<T>{};
      if (k0 + e * S::STEP < count && qn > 0) q[e] = some_quad(spot.at(base, ld, t0 + e * S::STEP), qn);
    }
  }
};

// A tile's rows of B or C in 32 bits, empty places zero.
template <class T, int LN>
__device__ __forceinline__ void stage_states(const T* base, int64_t ld, int lo, int count, int head,
                                             int N, float* to) {
  constexpr int NP = 4 * LN;
  for (int i = threadIdx.x; i < kSelTile * NP; i += kBlock) {
    const int t = i / NP, n = i % NP;
    to[i] = t < count && n < N ? load_one(base + (lo + (int64_t)t) * ld + (int64_t)head * N + n) : 0.f;
  }
}

// The step of a token: what comes in, its bias, softplus.
__device__ __forceinline__ float step_of(float v, float bias, int soft) {
  v += bias;
  return soft ? softplus(v) : v;
}

// The carry into a range from those before it (up: the gradient's, from those after it):
// the nearest one that does not pass its own carry on, then each one's whole decay and
// what it adds.
template <int LN>
__device__ __forceinline__ void carry_into(const SelCall& c, const SelPlan& p, int range, int dir,
                                           const SelPlace<LN>& w, const float (&A)[2][4],
                                           float (&h)[2][4]) {
  using S = SelShape<LN>;
  int j = range - dir;
  while (j - dir >= 0 && j - dir < p.ranges && p.info[j] == kSelOpen) j -= dir;
#pragma unroll
  for (int r = 0; r < S::RC; ++r)
#pragma unroll
    for (int k = 0; k < 4; ++k) h[r][k] = 0.f;
  for (; j != range; j += dir) {
#pragma unroll
    for (int r = 0; r < S::RC; ++r) {
      if (w.lane_c + r >= w.nc) continue;
      const int64_t at = (int64_t)j * c.D + w.c0 + w.lane_c + r;
      const float d = p.sums[at];
      const f4 s = ld4(p.states + at * S::NP + 4 * w.nl);
#pragma unroll
      for (int k = 0; k < 4; ++k) h[r][k] = __fmaf_rn(exp2_fast(d * A[r][k]), h[r][k], s[k]);
    }
  }
}

template <int LN>
__device__ __forceinline__ void load_rates(const SelCall& c, const SelPlace<LN>& w, float (&A)[2][4]) {
#pragma unroll
  for (int r = 0; r < 2; ++r) {
    const float* row = w.lane_c + r < w.nc ? c.A + (int64_t)(w.c0 + w.lane_c + r) * c.N : nullptr;
    load_states(row, c.N, w.nl, A[r]);
#pragma unroll
    for (int k = 0; k < 4; ++k) A[r][k] *= kLog2e;
  }
}

// A workgroup's tile in LDS.
template <int LN>
struct alignas(16) SelLds {
  using S = SelShape<LN>;
  float step[kSelTile * S::CB], dx[kSelTile * S::CB];
  float B[kSelTile * S::NP], C[kSelTile * S::NP];
  TileMarks marks;
  int from;
};

// ---------------------------------------------------------------- forward

// Where the first launch starts in a range: the start of the sequence that runs out of the
// range, the range's first token if that lies before it; hi if none runs out.
__device__ __forceinline__ int run_start(const Packed& s, int lo, int hi) {
  if (hi >= s.tokens) return hi;
  const int i = first_place(s, hi);  // the first offset >= hi
  if (i <= s.nseq && place_of(s, i) == hi) return hi;
  return i > 0 ? min(max(place_of(s, i - 1), lo), hi) : lo;
}
// ... and where the gradient's stops: the end of the sequence that runs into it.
__device__ __forceinline__ int run_stop(const Packed& s, int lo, int hi) {
  if (lo == 0) return lo;
  const int i = first_place(s, lo);
  if (i > s.nseq) return hi;
  const int o = place_of(s, i);
  return o == lo ? lo : max(min(o, hi), lo);
}

template <class T, int LN>
__global__ __launch_bounds__(kBlock) void k_selective_ends(SelCall c, SelPlan p) {
  using S = SelShape<LN>;
  __shared__ SelLds<LN> s;
  const int t = threadIdx.x;
  const int range = blockIdx.x / p.all_blocks, block = blockIdx.x % p.all_blocks;
  const SelPlace<LN> w(c, p, block);
  const int lo = range * p.range, hi = min(lo + p.range, c.seqs.tokens);
  if (t < kWave) {
    const int at = run_start(c.seqs, lo, hi);
    if (t == 0) s.from = at;
  }
  __syncthreads();
  const int from = s.from;
  // A sequence that starts in the range, or one that runs through all of it.
  const bool open = from == lo && lo > 0;
  int seq = -1;  // ... whose state before its first token counts, if it starts here
  bool starts = !open;
  if (open) {
    const int i = first_place(c.seqs, lo);
    starts = i <= c.seqs.nseq && place_of(c.seqs, i) == lo;
  }
  if (starts && from < hi) {  // the last offset <= from
    seq = first_place(c.seqs, from + 1) - 1;
    seq = max(0, min(seq, c.seqs.nseq - 1));
  }
  if (t == 0 && block == 0)
    p.info[range] = from == hi ? kSelNone : starts ? kSelClosed : kSelOpen;
  if (from == hi) return;

  float A[2][4], h[2][4], sum[2] = {0.f, 0.f};
  load_rates(c, w, A);
#pragma unroll
  for (int r = 0; r < 2; ++r) {
    const float* row = seq >= 0 && c.h0 && w.lane_c + r < w.nc
                           ? c.h0 + ((int64_t)seq * c.D + w.c0 + w.lane_c + r) * c.N
                           : nullptr;
    load_states(row, c.N, w.nl, h[r]);
  }
  float bias[4] = {0.f, 0.f, 0.f, 0.f};
  if (c.bias)
    for (int k = 0; k < w.qn; ++k) bias[k] = c.bias[w.q0 + k];
  const T* x = static_cast<const T*>(c.x);
  const T* delta = static_cast<const T*>(c.delta);
  const RowSpot xs = RowSpot::of(x, c.ld_x, w.k0, w.q0), ds = RowSpot::of(x, c.ld_delta, w.k0, w.q0);
  QuadTile<T, S> xn, dn;  // the next tile's
  const auto fetch = [&](int t0) {
    const int count = min(kSelTile, hi - t0);
    xn.load(x, c.ld_x, xs, t0, count, w.k0, w.qn);
    dn.load(delta, c.ld_delta, ds, t0, count, w.k0, w.qn);
  };
  fetch(from);

  for (int t0 = from; t0 < hi; t0 += kSelTile) {
    const int count = min(kSelTile, hi - t0);
    __syncthreads();
#pragma unroll
    for (int e = 0; e < S::EACH; ++e) {
      const int i = t + e * kBlock, k = w.k0 + e * S::STEP;
      if (k >= kSelTile) continue;
      float d[4], u[4];
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        d[j] = k < count && j < w.qn ? step_of(dn.q[e].get(j), bias[j], c.softplus) : 0.f;
        u[j] = d[j] * xn.q[e].get(j);
      }
      st4(s.step + i * 4, f4{d[0], d[1], d[2], d[3]});
      st4(s.dx + i * 4, f4{u[0], u[1], u[2], u[3]});
    }
    stage_states<T, LN>(static_cast<const T*>(c.B), c.ld_B, t0, count, w.head, c.N, s.B);
    if (t0 + kSelTile < hi) fetch(t0 + kSelTile);
    __syncthreads();
#pragma unroll 4
    for (int k = 0; k < kSelTile; ++k) {  // (tokens past the range: no step, nothing added)
      const float2 d = *reinterpret_cast<const float2*>(s.step + k * S::CB + w.lane_c);
      const float2 u = *reinterpret_cast<const float2*>(s.dx + k * S::CB + w.lane_c);
      const f4 B = ld4(s.B + k * S::NP + 4 * w.nl);
      const float dd[2] = {d.x, d.y}, uu[2] = {u.x, u.y};
#pragma unroll
      for (int r = 0; r < 2; ++r) {
        sum[r] += dd[r];
#pragma unroll
        for (int j = 0; j < 4; ++j)
          h[r][j] = __fmaf_rn(exp2_fast(dd[r] * A[r][j]), h[r][j], uu[r] * B[j]);
      }
    }
  }
#pragma unroll
  for (int r = 0; r < 2; ++r) {
    if (w.lane_c + r >= w.nc) continue;
    const int64_t at = (int64_t)range * c.D + w.c0 + w.lane_c + r;
    st4(p.states + at * S::NP + 4 * w.nl, f4{h[r][0], h[r][1], h[r][2], h[r][3]});
    if (w.nl == 0) p.sums[at] = sum[r];
  }
}

template <class T, int LN>
__global__ __launch_bounds__(kBlock) void k_selective(SelCall c, SelPlan p) {
  using S = SelShape<LN>;
  __shared__ SelLds<LN> s;
  __shared__ __align__(16) float sy[kSelTile * S::CB];
  __shared__ int list[kBlock];
  const int t = threadIdx.x;
  const int range = blockIdx.x / p.all_blocks, block = blockIdx.x % p.all_blocks;
  const SelPlace<LN> w(c, p, block);
  const int lo = range * p.range, hi = min(lo + p.range, c.seqs.tokens);

  // a lane's states of sequence i, before it or after it
  const auto row_of = [&](const float* base, int i, int r) -> float* {
    if (!base || w.lane_c + r >= w.nc) return nullptr;
    return const_cast<float*>(base) + ((int64_t)i * c.D + w.c0 + w.lane_c + r) * c.N;
  };
  check_places(c.seqs, range, p.ranges, c.last != nullptr, list, [&](int i) {
    for (int r = 0; r < 2; ++r) {
      float v[4];
      load_states(row_of(c.h0, i, r), c.N, w.nl, v);
      if (float* to = row_of(c.last, i, r)) store_states(to, c.N, w.nl, v);
    }
  });
  if (lo >= hi) return;

  const T* x = static_cast<const T*>(c.x);
  const T* delta = static_cast<const T*>(c.delta);
  const T* z = static_cast<const T*>(c.z);
  T* y = static_cast<T*>(c.y);
  const RowSpot xs = RowSpot::of(x, c.ld_x, w.k0, w.q0), ds = RowSpot::of(x, c.ld_delta, w.k0, w.q0);
  const RowSpot zs = RowSpot::of(x, c.ld_z, w.k0, w.q0), ys = RowSpot::of(x, c.ld_y, w.k0, w.q0);
  QuadTile<T, S> xn, dn, zn;  // the next tile's
  const auto fetch = [&](int t0) {
    const int count = min(kSelTile, hi - t0);
    xn.load(x, c.ld_x, xs, t0, count, w.k0, w.qn);
    dn.load(delta, c.ld_delta, ds, t0, count, w.k0, w.qn);
    if (c.z) zn.load(z, c.ld_z, zs, t0, count, w.k0, w.qn);
  };
  fetch(lo);
  float A[2][4], h[2][4];
  load_rates(c, w, A);
  float bias[4] = {0.f, 0.f, 0.f, 0.f}, skip[4] = {0.f, 0.f, 0.f, 0.f};
  for (int k = 0; k < w.qn; ++k) {
    if (c.bias) bias[k] = c.bias[w.q0 + k];
    if (c.skip) skip[k] = c.skip[w.q0 + k];
  }
  UpCursor cursor{};
  if (t < kWave) cursor.read(c.seqs, first_place(c.seqs, lo));

  for (int t0 = lo; t0 < hi; t0 += kSelTile) {
    const int count = min(kSelTile, hi - t0);
    const QuadTile<T, S> xv = xn, zv = zn;
#pragma unroll
    for (int e = 0; e < S::EACH; ++e) {
      const int i = t + e * kBlock, k = w.k0 + e * S::STEP;
      if (k >= kSelTile) continue;
      const bool there = k < count;
      float d[4], u[4];
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        d[j] = there && j < w.qn ? step_of(dn.q[e].get(j), bias[j], c.softplus) : 0.f;
        u[j] = d[j] * xv.q[e].get(j);
      }
      st4(s.step + i * 4, f4{d[0], d[1], d[2], d[3]});
      st4(s.dx + i * 4, f4{u[0], u[1], u[2], u[3]});
    }
    stage_states<T, LN>(static_cast<const T*>(c.B), c.ld_B, t0, count, w.head, c.N, s.B);
    stage_states<T, LN>(static_cast<const T*>(c.C), c.ld_C, t0, count, w.head, c.N, s.C);
    if (t < kWave) mark_tile(c.seqs, t0, t0 + count, cursor, s.marks);
    __syncthreads();
    const uint32_t starts = __builtin_amdgcn_readfirstlane(s.marks.starts);
    const uint32_t stops = __builtin_amdgcn_readfirstlane(s.marks.stops);
    if (t0 + kSelTile < hi) fetch(t0 + kSelTile);
    if (t0 == lo) {
      if (!(starts & 1) && lo > 0) {
        carry_into<LN>(c, p, range, 1, w, A, h);
      } else {
#pragma unroll
        for (int r = 0; r < 2; ++r)
#pragma unroll
          for (int j = 0; j < 4; ++j) h[r][j] = 0.f;
      }
    }
    if (c.marks) {
#pragma unroll
      for (int r = 0; r < 2; ++r) {
        if (w.lane_c + r >= w.nc || 4 * w.nl >= c.N) continue;
        const int64_t at = (int64_t)(t0 / kSelTile) * c.D + w.c0 + w.lane_c + r;
        st4(c.marks + at * p.NM + 4 * w.nl, f4{h[r][0], h[r][1], h[r][2], h[r][3]});
      }
    }
    const auto token = [&](int k) {
      const float2 d = *reinterpret_cast<const float2*>(s.step + k * S::CB + w.lane_c);
      const float2 u = *reinterpret_cast<const float2*>(s.dx + k * S::CB + w.lane_c);
      const f4 B = ld4(s.B + k * S::NP + 4 * w.nl), C = ld4(s.C + k * S::NP + 4 * w.nl);
      const float dd[2] = {d.x, d.y}, uu[2] = {u.x, u.y};
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
          const int from = __builtin_amdgcn_readfirstlane(s.marks.start[k]);
#pragma unroll
          for (int r = 0; r < 2; ++r) load_states(row_of(c.h0, from, r), c.N, w.nl, h[r]);
        }
        token(k);
        if ((stops >> k & 1) && c.last) {
          const int to = __builtin_amdgcn_readfirstlane(s.marks.stop[k]);
#pragma unroll
          for (int r = 0; r < 2; ++r)
            if (float* row = row_of(c.last, to, r)) store_states(row, c.N, w.nl, h[r]);
        }
      }
    }
    __syncthreads();
#pragma unroll
    for (int e = 0; e < S::EACH; ++e) {
      const int i = t + e * kBlock, k = w.k0 + e * S::STEP;
      if (k >= count || w.qn <= 0) continue;
      const f4 q = ld4(sy + i * 4);
      float v[4] = {q[0], q[1], q[2], q[3]};
      if (c.skip) {
#pragma unroll
        for (int j = 0; j < 4; ++j) v[j] = __fmaf_rn(skip[j], xv.q[e].get(j), q[j]);
      }
      if (c.z) {
#pragma unroll
        for (int j = 0; j < 4; ++j) v[j] *= zv.q[e].get(j) * sigmoid(zv.q[e].get(j));
      }
      put_quad(ys.at(y, c.ld_y, t0 + e * S::STEP), v, w.qn);
    }
  }
}

// One token for each sequence: LN lanes of four states each for a channel of a row.
template <class T, int LN>
__global__ __launch_bounds__(kBlock) void k_selective_step(SelCall c, int blocks) {
  constexpr int CB = kBlock / LN;  // channels of a workgroup
  const int nl = threadIdx.x % LN;
  const int64_t all = (int64_t)c.seqs.nseq * blocks;
  for (int64_t i = blockIdx.x; i < all; i += gridDim.x) {
    const int64_t row = i / blocks;
    const int ch = (int)(i - row * blocks) * CB + threadIdx.x / LN;
    const bool live = ch < c.D;
    const int own = live ? ch : 0, head = own / (c.D / c.groups);
    const int64_t at = (row * c.D + own) * c.N;
    const T* B = static_cast<const T*>(c.B) + row * c.ld_B + (int64_t)head * c.N;
    const T* C = static_cast<const T*>(c.C) + row * c.ld_C + (int64_t)head * c.N;
    const float x = load_one(static_cast<const T*>(c.x) + row * c.ld_x + own);
    const float raw = load_one(static_cast<const T*>(c.delta) + row * c.ld_delta + own);
    float A[4], h[4], Bv[4], Cv[4];
    load_states(c.A + (int64_t)own * c.N, c.N, nl, A);
    load_states(c.h0 ? c.h0 + at : nullptr, c.N, nl, h);
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      const int n = 4 * nl + j;
      Bv[j] = n < c.N ? load_one(B + n) : 0.f;
      Cv[j] = n < c.N ? load_one(C + n) : 0.f;
    }
    const float d = step_of(raw, c.bias ? c.bias[own] : 0.f, c.softplus), u = d * x;
    float v = 0.f;
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      h[j] = __fmaf_rn(exp2_fast(d * (A[j] * kLog2e)), h[j], u * Bv[j]);
      v = __fmaf_rn(Cv[j], h[j], v);
    }
    v = sum_states<LN>(v);
    if (!live) continue;
    if (c.last) store_states(c.last + at, c.N, nl, h);
    if (nl == 0) {
      if (c.skip) v = __fmaf_rn(c.skip[own], x, v);
      if (c.z) {
        const float z = load_one(static_cast<const T*>(c.z) + row * c.ld_z + own);
        v *= z * sigmoid(z);
      }
      static_cast<T*>(c.y)[row * c.ld_y + own] = Elem<T>::put(settled(v));
    }
  }
}

}  // namespace pg
