// Short causal convolution of every channel over packed sequences, and its gradient:
//   u_t[c] = bias[c] + sum_{k < K} w[c][k] x_{t-K+1+k}[c],   y = u or u sigmoid(u)
// where a sequence's first tokens reach back into its state, the K - 1 inputs before it.
//
// A thread takes four channels of a run of consecutive tokens and keeps the last K - 1
// inputs in registers: every tensor is read once and written once, but for the K - 1
// tokens before a run (the gradient: behind it, too), which the caches hold.
// The gradient walks forward as well: a token's g = dy act'(u) goes into K sums, for itself
// and the K - 1 inputs before it; the oldest of them is complete and leaves.
#pragma once
#include "selective_dev.h"

namespace pg {

constexpr int kConvRoom = kBlock / kConvMinLanes * kConvRun + kConvMaxK;  // marked places

struct ConvLds {
  int start[kConvRoom], stop[kConvRoom];
  int before[kWave];  // the sequence of the token before each 64th of the tile
  int list[kBlock];
};

// The places of a tile of `tokens` tokens (a multiple of 64), and K - 1 more, by wave 0.
__device__ __forceinline__ void conv_places(const Packed& s, int lo, int tokens, int more,
                                            ConvLds& l) {
  const int lane = lane_id();
  const int hi = (int)min((int64_t)lo + tokens + more, (int64_t)s.tokens);
  const int cursor = first_place(s, lo);
  mark_places(s, lo, hi, tokens + more, cursor, l.start, l.stop);
  const int seg = tokens / kWave;
  int m = -1;
  for (int j = 0; j < seg; ++j) m = max(m, l.start[lane * seg + j]);
#pragma unroll
  for (int d = 1; d < kWave; d *= 2) {
    const int o = __shfl_up(m, d);
    if (lane >= d) m = max(m, o);
  }
  const int o = __shfl_up(m, 1);
  l.before[lane] = min(s.nseq - 1, max(0, max(lane ? o : -1, cursor - 1)));
}

// A thread's tile, run and channels.
struct ConvPlace {
  int cl, tl, ch, nv;
  __device__ __forceinline__ ConvPlace(const ConvCall& c, int block) {
    const int CT = 1 << c.lanes_log2;
    cl = threadIdx.x & (CT - 1);
    tl = threadIdx.x >> c.lanes_log2;
    ch = (block * CT + cl) * 4;
    nv = max(0, min(4, c.D - ch));
    if (nv == 0) ch = 0;
  }
};

template <class T>
__device__ __forceinline__ void conv_state(const ConvCall& c, const void* state, int K, int seq, int row,
                                           const ConvPlace& w, float (&v)[4]) {
  Quad<T> q{};
  if (state && w.nv > 0)
    q = some_quad(static_cast<const T*>(state) + ((int64_t)seq * (K - 1) + row) * c.D + w.ch, w.nv);
#pragma unroll
  for (int j = 0; j < 4; ++j) v[j] = q.get(j);
}

// Copies an empty sequence's rows, the workgroup's channels of them.
template <class T>
__device__ __forceinline__ void conv_copy(const ConvCall& c, int K, int seq, const void* from, void* to,
                                          const ConvPlace& w) {
  if (w.nv <= 0) return;
  for (int row = w.tl; row < K - 1; row += kBlock >> c.lanes_log2) {
    float v[4];
    conv_state<T>(c, from, K, seq, row, w, v);
    put_quad(static_cast<T*>(to) + ((int64_t)seq * (K - 1) + row) * c.D + w.ch, v, w.nv);
  }
}

template <int K>
__device__ __forceinline__ void conv_weights(const ConvCall& c, const ConvPlace& w, float (&wt)[K][4],
                                             float (&bias)[4]) {
#pragma unroll
  for (int j = 0; j < 4; ++j) {
    const bool there = j < w.nv;
    bias[j] = there && c.bias ? c.bias[w.ch + j] : 0.f;
#pragma unroll
    for (int k = 0; k < K; ++k) wt[k][j] = there ? c.weight[(int64_t)(w.ch + j) * K + k] : 0.f;
  }
}

// The inputs before token t of sequence seq, `place` tokens into it.
template <class T, int K>
__device__ __forceinline__ void conv_window(const ConvCall& c, const ConvPlace& w, int t, int seq, int place,
                                            float (&win)[K][4]) {
#pragma unroll
  for (int k = 0; k < K - 1; ++k) {
    const int back = K - 1 - k;
    if (place >= back) {
      Quad<T> q{};
      if (w.nv > 0) q = some_quad(static_cast<const T*>(c.x) + (t - (int64_t)back) * c.ld_x + w.ch, w.nv);
#pragma unroll
      for (int j = 0; j < 4; ++j) win[k][j] = q.get(j);
    } else {
      conv_state<T>(c, c.state, K, seq, K - 1 + place - back, w, win[k]);
    }
  }
}

template <int K>
__device__ __forceinline__ void conv_sum(const float (&wt)[K][4], const float (&bias)[4],
                                         const float (&win)[K][4], float (&u)[4]) {
#pragma unroll
  for (int j = 0; j < 4; ++j) {
    u[j] = bias[j];
#pragma unroll
    for (int k = 0; k < K; ++k) u[j] = __fmaf_rn(wt[k][j], win[k][j], u[j]);
  }
}

template <class T, int K>
__global__ __launch_bounds__(kBlock) void k_convolution(ConvCall c) {
  constexpr int R = kConvRun;
  __shared__ ConvLds l;
  const int t = threadIdx.x;
  const int tile = blockIdx.x / c.blocks, block = blockIdx.x % c.blocks;
  const ConvPlace w(c, block);
  const int tokens = (kBlock >> c.lanes_log2) * R;
  const int lo = tile * tokens;
  check_places(c.seqs, tile, c.tiles, kBlock, c.last != nullptr && K > 1, l.list,
               [&](int i) { conv_copy<T>(c, K, i, c.state, c.last, w); });
  if (lo >= c.seqs.tokens) return;
  const int t0 = lo + w.tl * R, count = max(0, min(R, c.seqs.tokens - t0));
  const T* x = static_cast<const T*>(c.x) + w.ch;
  Quad<T> xv[R];
#pragma unroll
  for (int i = 0; i < R; ++i) {
    xv[i] = Quad<T>{};
    if (i < count && w.nv > 0) xv[i] = some_quad(x + (t0 + (int64_t)i) * c.ld_x, w.nv);
  }
  float wt[K][4], bias[4], win[K][4];
  conv_weights<K>(c, w, wt, bias);
  if (t < kWave) conv_places(c.seqs, lo, tokens, 0, l);
  __syncthreads();
  if (count == 0 || w.nv == 0) return;
  int seq = l.before[w.tl * R / (tokens / kWave)];
  if (l.start[t0 - lo] < 0) conv_window<T, K>(c, w, t0, seq, max(0, t0 - place_of(c.seqs, seq)), win);
#pragma unroll
  for (int i = 0; i < R; ++i) {
    if (i >= count) continue;
    const int from = l.start[t0 - lo + i];
    if (from >= 0) {
      seq = from;
      conv_window<T, K>(c, w, t0 + i, seq, 0, win);
    }
#pragma unroll
    for (int j = 0; j < 4; ++j) win[K - 1][j] = xv[i].get(j);
    float u[4];
    conv_sum<K>(wt, bias, win, u);
    if (c.silu) {
#pragma unroll
      for (int j = 0; j < 4; ++j) u[j] *= sigmoid(u[j]);
    }
    put_quad(static_cast<T*>(c.y) + (t0 + (int64_t)i) * c.ld_y + w.ch, u, w.nv);
    if (c.last && l.stop[t0 - lo + i] >= 0) {
#pragma unroll
      for (int k = 1; k < K; ++k)
        put_quad(static_cast<T*>(c.last) + ((int64_t)seq * (K - 1) + k - 1) * c.D + w.ch, win[k], w.nv);
    }
#pragma unroll
    for (int k = 0; k < K - 1; ++k)
#pragma unroll
      for (int j = 0; j < 4; ++j) win[k][j] = win[k + 1][j];
  }
}

// One token for each sequence; a thread reads all that it needs before it writes.
template <class T, int K>
__global__ __launch_bounds__(kBlock) void k_convolution_step(ConvCall c) {
  const int quads = ceil_div(c.D, 4);
  const int64_t all = (int64_t)c.seqs.nseq * quads;
  for (int64_t i = (int64_t)blockIdx.x * kBlock + threadIdx.x; i < all; i += (int64_t)gridDim.x * kBlock) {
    const int row = (int)(i / quads);
    ConvPlace w(c, 0);
    w.ch = (int)(i % quads) * 4;
    w.nv = min(4, c.D - w.ch);
    float wt[K][4], bias[4], win[K][4], u[4];
#pragma unroll
    for (int k = 0; k < K - 1; ++k) conv_state<T>(c, c.state, K, row, k, w, win[k]);
    const Quad<T> xv = some_quad(static_cast<const T*>(c.x) + row * c.ld_x + w.ch, w.nv);
    conv_weights<K>(c, w, wt, bias);
#pragma unroll
    for (int j = 0; j < 4; ++j) win[K - 1][j] = xv.get(j);
    conv_sum<K>(wt, bias, win, u);
    if (c.silu) {
#pragma unroll
      for (int j = 0; j < 4; ++j) u[j] *= sigmoid(u[j]);
    }
    put_quad(static_cast<T*>(c.y) + row * c.ld_y + w.ch, u, w.nv);
    if (c.last) {
#pragma unroll
      for (int k = 1; k < K; ++k)
        put_quad(static_cast<T*>(c.last) + ((int64_t)row * (K - 1) + k - 1) * c.D + w.ch, win[k], w.nv);
    }
  }
}

template <class T, int K>
__global__ __launch_bounds__(kBlock) void k_convolution_grad(ConvCall c) {
  constexpr int R = kConvRun;
  __shared__ ConvLds l;
  __shared__ __align__(16) float red[kBlock * 4];
  const int t = threadIdx.x;
  const int group = blockIdx.x / c.blocks, block = blockIdx.x % c.blocks;
  const ConvPlace w(c, block);
  const int CT = 1 << c.lanes_log2, TL = kBlock >> c.lanes_log2, tokens = TL * R;
  check_places(c.seqs, group, c.groups, kBlock, c.dstate != nullptr && K > 1, l.list,
               [&](int i) { conv_copy<T>(c, K, i, c.dlast, c.dstate, w); });
  float wt[K][4], bias[4], dw[K][4], db[4] = {0.f, 0.f, 0.f, 0.f};
  conv_weights<K>(c, w, wt, bias);
#pragma unroll
  for (int k = 0; k < K; ++k)
#pragma unroll
    for (int j = 0; j < 4; ++j) dw[k][j] = 0.f;

  for (int tile = group; tile < c.tiles; tile += c.groups) {
    const int lo = tile * tokens;
    __syncthreads();
    if (t < kWave) conv_places(c.seqs, lo, tokens, K - 1, l);
    __syncthreads();
    const int t0 = lo + w.tl * R;
    if (t0 >= c.seqs.tokens || w.nv == 0) continue;
    const int end = (int)min((int64_t)t0 + R + K - 1, (int64_t)c.seqs.tokens);  // looked at
    float win[K][4], acc[K][4];
#pragma unroll
    for (int k = 0; k < K; ++k)
#pragma unroll
      for (int j = 0; j < 4; ++j) acc[k][j] = 0.f;
    int seq = l.before[w.tl * R / (tokens / kWave)], place = 0;
    if (l.start[t0 - lo] < 0) {
      place = max(0, t0 - place_of(c.seqs, seq));
      conv_window<T, K>(c, w, t0, seq, place, win);
    }
    for (int at = t0; at < end; ++at) {
      const int from = l.start[at - lo];
      if (from >= 0) {
        if (at >= t0 + R) break;  // the run's last sequence has ended
        seq = from;
        place = 0;
        conv_window<T, K>(c, w, at, seq, 0, win);
      }
      const Quad<T> xv = some_quad(static_cast<const T*>(c.x) + (int64_t)at * c.ld_x + w.ch, w.nv);
      const Quad<T> gv = some_quad(static_cast<const T*>(c.dy) + (int64_t)at * c.ld_dy + w.ch, w.nv);
      float g[4];
#pragma unroll
      for (int j = 0; j < 4; ++j) win[K - 1][j] = xv.get(j), g[j] = gv.get(j);
      if (c.silu) {
        float u[4];
        conv_sum<K>(wt, bias, win, u);
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          const float s = sigmoid(u[j]);
          g[j] *= s * __fmaf_rn(u[j], 1.f - s, 1.f);
        }
      }
      if (at < t0 + R) {
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          db[j] += g[j];
#pragma unroll
          for (int k = 0; k < K; ++k) dw[k][j] = __fmaf_rn(g[j], win[k][j], dw[k][j]);
        }
      }
#pragma unroll
      for (int b = 0; b < K; ++b)
#pragma unroll
        for (int j = 0; j < 4; ++j) acc[b][j] = __fmaf_rn(wt[K - 1 - b][j], g[j], acc[b][j]);
      // What is complete leaves: the input b tokens back, or that row of the state.
      const auto emit = [&](int b, const float (&v)[4]) {
        if (place >= b) {
          const int s = at - b;
          if (s >= t0 && s < t0 + R) put_quad(static_cast<T*>(c.dx) + (int64_t)s * c.ld_dx + w.ch, v, w.nv);
        } else if (c.dstate && at - place >= t0 && at - place < t0 + R) {
          put_quad(static_cast<T*>(c.dstate) + ((int64_t)seq * (K - 1) + K - 1 + place - b) * c.D + w.ch, v,
                   w.nv);
        }
      };
      if (l.stop[at - lo] >= 0) {
#pragma unroll
        for (int b = K - 1; b >= 0; --b) {
          float v[4] = {acc[b][0], acc[b][1], acc[b][2], acc[b][3]};
          if (b < K - 1 && c.dlast) {
            float d[4];
            conv_state<T>(c, c.dlast, K, seq, K - 2 - b, w, d);
#pragma unroll
            for (int j = 0; j < 4; ++j) v[j] += d[j];
          }
          emit(b, v);
#pragma unroll
          for (int j = 0; j < 4; ++j) acc[b][j] = 0.f;
        }
      } else {
        emit(K - 1, acc[K - 1]);
#pragma unroll
        for (int b = K - 1; b > 0; --b)
#pragma unroll
          for (int j = 0; j < 4; ++j) acc[b][j] = acc[b - 1][j];
#pragma unroll
        for (int j = 0; j < 4; ++j) acc[0][j] = 0.f;
      }
#pragma unroll
      for (int k = 0; k < K - 1; ++k)
#pragma unroll
        for (int j = 0; j < 4; ++j) win[k][j] = win[k + 1][j];
      ++place;
    }
  }

  // the workgroup's runs, in order
#pragma unroll
  for (int k = 0; k <= K; ++k) {
    __syncthreads();
    if (k < K) st4(red + t * 4, f4{dw[k < K ? k : 0][0], dw[k < K ? k : 0][1], dw[k < K ? k : 0][2], dw[k < K ? k : 0][3]});
    else st4(red + t * 4, f4{db[0], db[1], db[2], db[3]});
    __syncthreads();
    const int ch = block * 4 * CT + t;
    if (t < 4 * CT && ch < c.D) {
      float v = 0.f;
      for (int j = 0; j < TL; ++j) v += red[j * 4 * CT + t];
      c.part[((int64_t)group * (K + 1) + k) * c.D + ch] = v;
    }
  }
}

// dw and the bias's gradient from the groups' sums: 64 of them to a workgroup, a quarter of
// the groups to each thread.
__global__ __launch_bounds__(kBlock) void k_convolution_sums(ConvCall c, int K) {
  __shared__ float part[kBlock];
  const int t = threadIdx.x;
  const int64_t o = (int64_t)blockIdx.x * kWave + t % kWave, all = (int64_t)(K + 1) * c.D;
  float v = 0.f;
  if (o < all) {
#pragma unroll 8
    for (int g = t / kWave; g < c.groups; g += kWavesPerBlock) v += c.part[g * all + o];
  }
  part[t] = v;
  __syncthreads();
  if (t >= kWave || o >= all) return;
  v = (part[t] + part[t + 64]) + (part[t + 128] + part[t + 192]);
  const int64_t k = o / c.D, ch = o % c.D;
  if (k < K) c.dweight[ch * K + k] = v;
  else if (c.dbias) c.dbias[ch] = v;
}

}  // namespace pg
