// Short causal convolution of every channel over packed sequences, and its gradient:
//   u_t[c] = bias[c] + sum_{k < K} w[c][k] x_{t-K+1+k}[c],   y = u or u sigmoid(u)
// where a sequence's first tokens reach back into its state, the K - 1 inputs before it.
//
// A row of lanes takes a chunk of consecutive tokens, four or eight channels to a lane, and
// goes through it in steps of eight tokens with the last K - 1 inputs in registers and the
// next step's inputs on their way: every tensor is read once and written once, but for the
// K - 1 tokens before a chunk (the gradient: behind it, too).  Which sequence it is in and
// where that ends, it keeps; no two waves wait for each other.  The gradient walks forward as
// well: a token's g = dy act'(u) goes into K sums, for itself and the K - 1 inputs before it;
// the oldest of them is complete and leaves.
//
// What bounds it is memory: 65,536 x 2,048 bfloat16 in 16 sequences, K 4, take 120 us forward
// (537 MB, 4.5 TB/s; a copy of 1 GiB reaches 5.2) and 198 in the gradient (805 MB, 4.1).  Tiles
// in LDS with barriers for the sequences' marks took 156; eight channels to a lane read 16
// bytes at a time.
#pragma once
#include <type_traits>

#include "selective_dev.h"

namespace pg {

// f(0), ..., f(N - 1), each by itself: loads held in registers are indexed by constants.
template <int N, class F>
__device__ __forceinline__ void each(F f) {
  if constexpr (N > 0) {
    each<N - 1>(f);
    f(std::integral_constant<int, N - 1>{});
  }
}

// The sequence that a row of lanes is in, and where that ends.
struct ConvWalk {
  int seq, end;
  // The one that token t lies in: the last offset <= t, found by the row's lanes side by side.
  __device__ __forceinline__ ConvWalk(const Packed& s, int t, int lanes_log2) {
    const int lanes = 1 << lanes_log2, l = lane_id() & (lanes - 1), row = lane_id() >> lanes_log2;
    int at = 0, n = s.nseq + 1;  // the first offset > t is in [at, at + n]
    while (__ballot(n > 0)) {
      const int step = ceil_div(n, lanes + 1);
      const int i = at + (l + 1) * step - 1;
      const bool below = n > 0 && i < at + n && place_of(s, i) <= t;
      const uint64_t all = __ballot(below) >> (row << lanes_log2);
      const int k = __popcll(lanes == kWave ? all : all & ((1ull << lanes) - 1));
      at += k * step;
      n -= k * step;
      if (k < lanes) n = min(max(step - 1, 0), n);
    }
    seq = min(max(at - 1, 0), s.nseq - 1);
    end = place_of(s, seq + 1);
  }
  // To the next sequence that has tokens, if token t is its first.
  __device__ __forceinline__ bool next(const Packed& s, int t) {
    if (t != end) return false;
    do {
      end = ++seq < s.nseq ? place_of(s, seq + 1) : INT32_MAX;
    } while (end <= t);
    seq = min(seq, s.nseq - 1);
    return true;
  }
};

// V channels in 8 or 16 bytes, any alignment; at a row's end the first n of them.
template <class T, int V>
struct Strip {
  typedef std::conditional_t<V * sizeof(T) == 16, u4_any, u2_any> Raw;
  Raw raw;
  __device__ __forceinline__ float get(int i) const {
    if constexpr (sizeof(T) == 4) return __uint_as_float(raw[i]);
    else return Elem<T>::get(T{(uint16_t)(i & 1 ? raw[i / 2] >> 16 : raw[i / 2])});
  }
  __device__ __forceinline__ void load(const T* p, int n) {
    raw = Raw{};
    if (n == V) {
      raw = *reinterpret_cast<const Raw*>(p);
    } else {
#pragma unroll
      for (int i = 0; i < V - 1; ++i) {
        if (i >= n) continue;
        if constexpr (sizeof(T) == 4) raw[i] = __float_as_uint(p[i]);
        else raw[i / 2] |= (uint32_t)p[i].bits << (16 * (i & 1));
      }
    }
  }
  static __device__ __forceinline__ void store(T* p, const float (&v)[V], int n) {
    if (n == V) {
      if constexpr (V == 4) store_quad<T, true>(p, v, 4);
      else Oct<T>::store(p, v);
    } else {
#pragma unroll
      for (int i = 0; i < V - 1; ++i)
        if (i < n) p[i] = Elem<T>::put(settled(v[i]));
    }
  }
};

// A thread's chunk and channels.  The last lane of a row takes whole strips, too, where the
// row has one: it starts `shift` channels early, and its neighbour computes and writes the
// same values there.
template <int V>
struct ConvPlace {
  int cl, tl, ch, nv, shift;
  __device__ __forceinline__ ConvPlace(const ConvCall& c, int block) {
    const int CT = 1 << c.lanes_log2;
    cl = threadIdx.x & (CT - 1);
    tl = threadIdx.x >> c.lanes_log2;
    ch = (block * CT + cl) * V;
    nv = max(0, min(V, c.D - ch));
    shift = 0;
    if (nv == 0) {
      ch = 0;
    } else if (nv < V && c.D >= V) {
      shift = V - nv;
      ch -= shift;
      nv = V;
    }
  }
};

// A row of a sequence's state (none: zeros).
template <class T, int V>
__device__ __forceinline__ void conv_state(const ConvCall& c, const void* state, int K, int seq, int row,
                                           const ConvPlace<V>& w, float (&v)[V]) {
  Strip<T, V> q;
  q.load(static_cast<const T*>(state) + ((int64_t)seq * (K - 1) + row) * c.D + w.ch, state ? w.nv : 0);
#pragma unroll
  for (int j = 0; j < V; ++j) v[j] = q.get(j);
}

// Copies an empty sequence's rows, the workgroup's channels of them.
template <class T, int V>
__device__ __forceinline__ void conv_copy(const ConvCall& c, int K, int seq, const void* from, void* to,
                                          const ConvPlace<V>& w) {
  if (w.nv <= 0) return;
  for (int row = w.tl; row < K - 1; row += kBlock >> c.lanes_log2) {
    float v[V];
    conv_state<T>(c, from, K, seq, row, w, v);
    Strip<T, V>::store(static_cast<T*>(to) + ((int64_t)seq * (K - 1) + row) * c.D + w.ch, v, w.nv);
  }
}

template <int K, int V>
__device__ __forceinline__ void conv_weights(const ConvCall& c, const ConvPlace<V>& w, float (&wt)[K][V],
                                             float (&bias)[V]) {
  struct __attribute__((packed, aligned(4))) Taps {
    float k[K];
  };
  const Taps* rows = reinterpret_cast<const Taps*>(c.weight) + w.ch;
#pragma unroll
  for (int j = 0; j < V; ++j) {
    Taps q{};
    if (j < w.nv) q = rows[j];
#pragma unroll
    for (int k = 0; k < K; ++k) wt[k][j] = q.k[k];
    bias[j] = j < w.nv && c.bias ? c.bias[w.ch + j] : 0.f;
  }
}

// The inputs before token t of sequence seq, `place` tokens into it.
template <class T, int K, int V>
__device__ __forceinline__ void conv_window(const ConvCall& c, const ConvPlace<V>& w, int t, int seq, int place,
                                            float (&win)[K][V]) {
#pragma unroll
  for (int k = 0; k < K - 1; ++k) {
    const int back = K - 1 - k;
    if (place >= back) {
      Strip<T, V> q;
      q.load(static_cast<const T*>(c.x) + (t - (int64_t)back) * c.ld_x + w.ch, w.nv);
#pragma unroll
      for (int j = 0; j < V; ++j) win[k][j] = q.get(j);
    } else {
      conv_state<T>(c, c.state, K, seq, K - 1 + place - back, w, win[k]);
    }
  }
}

template <int K, int V>
__device__ __forceinline__ void conv_sum(const float (&wt)[K][V], const float (&bias)[V],
                                         const float (&win)[K][V], float (&u)[V]) {
#pragma unroll
  for (int j = 0; j < V; ++j) {
    u[j] = bias[j];
#pragma unroll
    for (int k = 0; k < K; ++k) u[j] = __fmaf_rn(wt[k][j], win[k][j], u[j]);
  }
}
template <int K, int V>
__device__ __forceinline__ void conv_shift(float (&win)[K][V]) {
#pragma unroll
  for (int k = 0; k < K - 1; ++k)
#pragma unroll
    for (int j = 0; j < V; ++j) win[k][j] = win[k + 1][j];
}

template <class T, int K, int V>
__global__ __launch_bounds__(kBlock) void k_convolution(ConvCall c) {
  constexpr int R = kConvStep;
  __shared__ int list[kBlock + 1];
  const int group = blockIdx.x / c.blocks, block = blockIdx.x % c.blocks;
  const ConvPlace<V> w(c, block);
  check_places(c.seqs, group, c.groups, kBlock, c.last != nullptr && K > 1, list,
               [&](int i) { conv_copy<T>(c, K, i, c.state, c.last, w); });
  const int64_t chunk = (int64_t)group * (kBlock >> c.lanes_log2) + w.tl;
  const int t0 = (int)min(chunk * c.chunk, (int64_t)c.seqs.tokens);
  const int t1 = (int)min((int64_t)t0 + c.chunk, (int64_t)c.seqs.tokens);
  const T* x = static_cast<const T*>(c.x) + w.ch;
  T* y = static_cast<T*>(c.y) + w.ch;
  Strip<T, V> xv[R];
  const auto fetch = [&](int at) {
#pragma unroll
    for (int i = 0; i < R; ++i) xv[i].load(x + (at + (int64_t)i) * c.ld_x, at + i < t1 ? w.nv : 0);
  };
  fetch(t0);
  float wt[K][V], bias[V], win[K][V];
  conv_weights<K>(c, w, wt, bias);
  ConvWalk walk(c.seqs, min(t0, c.seqs.tokens - 1), c.lanes_log2);
  if (t0 >= t1 || w.nv == 0) return;
  conv_window<T, K>(c, w, t0, walk.seq, max(0, t0 - place_of(c.seqs, walk.seq)), win);
  const auto token = [&](const Strip<T, V>& in, T* to) {
#pragma unroll
    for (int j = 0; j < V; ++j) win[K - 1][j] = in.get(j);
    float u[V];
    conv_sum<K>(wt, bias, win, u);
    if (c.silu) {
#pragma unroll
      for (int j = 0; j < V; ++j) u[j] *= sigmoid(u[j]);
    }
    Strip<T, V>::store(to, u, w.nv);
  };
  for (int at = t0; at < t1; at += R) {
    Strip<T, V> now[R];
#pragma unroll
    for (int i = 0; i < R; ++i) now[i] = xv[i];
    if (at + R < t1) fetch(at + R);
    T* to = y + (int64_t)at * c.ld_y;
    if (walk.end > at + R && at + R <= t1) {  // the usual step, in the middle of a sequence
      each<R>([&](auto step) {
        constexpr int i = decltype(step)::value;
        token(now[i], to + i * c.ld_y);
        conv_shift<K>(win);
      });
      continue;
    }
    each<R>([&](auto step) {
      constexpr int i = decltype(step)::value;
      const int k = at + i;
      if (k >= t1) return;
      if (walk.next(c.seqs, k)) conv_window<T, K>(c, w, k, walk.seq, 0, win);
      token(now[i], to + i * c.ld_y);
      if (c.last && k + 1 == walk.end) {
#pragma unroll
        for (int j = 1; j < K; ++j)
          Strip<T, V>::store(static_cast<T*>(c.last) + ((int64_t)walk.seq * (K - 1) + j - 1) * c.D + w.ch, win[j],
                             w.nv);
      }
      conv_shift<K>(win);
    });
  }
}

// One token for each sequence; a thread reads all that it needs before it writes.  64 x 512
// takes 3.4 us, a launch and one round trip of loads.
template <class T, int K, int V>
__global__ __launch_bounds__(kBlock) void k_convolution_step(ConvCall c) {
  const int strips = ceil_div(c.D, V);
  const int64_t all = (int64_t)c.seqs.nseq * strips;
  for (int64_t i = (int64_t)blockIdx.x * kBlock + threadIdx.x; i < all; i += (int64_t)gridDim.x * kBlock) {
    const int row = (int)(i / strips);
    ConvPlace<V> w(c, 0);  // (last may be state: no channel twice)
    w.ch = (int)(i % strips) * V;
    w.nv = min(V, c.D - w.ch);
    float wt[K][V], bias[V], win[K][V], u[V];
#pragma unroll
    for (int k = 0; k < K - 1; ++k) conv_state<T>(c, c.state, K, row, k, w, win[k]);
    Strip<T, V> xv;
    xv.load(static_cast<const T*>(c.x) + row * c.ld_x + w.ch, w.nv);
    conv_weights<K>(c, w, wt, bias);
#pragma unroll
    for (int j = 0; j < V; ++j) win[K - 1][j] = xv.get(j);
    conv_sum<K>(wt, bias, win, u);
    if (c.silu) {
#pragma unroll
      for (int j = 0; j < V; ++j) u[j] *= sigmoid(u[j]);
    }
    Strip<T, V>::store(static_cast<T*>(c.y) + row * c.ld_y + w.ch, u, w.nv);
    if (c.last) {
#pragma unroll
      for (int k = 1; k < K; ++k)
        Strip<T, V>::store(static_cast<T*>(c.last) + ((int64_t)row * (K - 1) + k - 1) * c.D + w.ch, win[k], w.nv);
    }
  }
}

// Four tokens ahead, not eight: x and dy of each, with the sums of K taps, are 130 to 175
// registers.  16,411 x 255 float32 in 700 sequences, K 3: 19 us and 4 for the sums, where the
// bytes are 10; four steps of four tokens to a row, then the join of the workgroup's sums.
template <class T, int K, int V>
__global__ __launch_bounds__(kBlock, conv_grad_waves(sizeof(T))) void k_convolution_grad(ConvCall c) {
  constexpr int R = kConvStep / 2;
  __shared__ int list[kBlock + 1];
  __shared__ __align__(16) float red[kBlock * V];
  const int t = threadIdx.x;
  const int group = blockIdx.x / c.blocks, block = blockIdx.x % c.blocks;
  const ConvPlace<V> w(c, block);
  const int CT = 1 << c.lanes_log2, TL = kBlock >> c.lanes_log2;
  check_places(c.seqs, group, c.groups, kBlock, c.dstate != nullptr && K > 1, list,
               [&](int i) { conv_copy<T>(c, K, i, c.dlast, c.dstate, w); });
  const int64_t chunk = (int64_t)group * TL + w.tl;
  const int t0 = (int)min(chunk * c.chunk, (int64_t)c.seqs.tokens);
  const int t1 = (int)min((int64_t)t0 + c.chunk, (int64_t)c.seqs.tokens);
  const int end = (int)min((int64_t)t1 + K - 1, (int64_t)c.seqs.tokens);  // looked at
  const T* x = static_cast<const T*>(c.x) + w.ch;
  const T* dy = static_cast<const T*>(c.dy) + w.ch;
  T* dx = static_cast<T*>(c.dx) + w.ch;
  Strip<T, V> xv[R], gv[R];
  const auto fetch = [&](int at) {
#pragma unroll
    for (int i = 0; i < R; ++i) {
      xv[i].load(x + (at + (int64_t)i) * c.ld_x, at + i < end ? w.nv : 0);
      gv[i].load(dy + (at + (int64_t)i) * c.ld_dy, at + i < end ? w.nv : 0);
    }
  };
  fetch(t0);
  float wt[K][V], bias[V], dw[K][V], db[V], win[K][V], acc[K][V];
  conv_weights<K>(c, w, wt, bias);
#pragma unroll
  for (int j = 0; j < V; ++j) {
    db[j] = 0.f;
#pragma unroll
    for (int k = 0; k < K; ++k) dw[k][j] = acc[k][j] = 0.f;
  }
  ConvWalk walk(c.seqs, min(t0, max(0, c.seqs.tokens - 1)), c.lanes_log2);
  if (t0 < t1 && w.nv > 0) {
    int begin = min(place_of(c.seqs, walk.seq), t0);  // of the sequence
    conv_window<T, K>(c, w, t0, walk.seq, t0 - begin, win);
    // A token's g into the sums: own, of the chunk (not of those looked at behind it).
    const auto take = [&](const Strip<T, V>& xi, const Strip<T, V>& gi, bool own) {
      float g[V];
#pragma unroll
      for (int j = 0; j < V; ++j) win[K - 1][j] = xi.get(j), g[j] = gi.get(j);
      if (c.silu) {
        float u[V];
        conv_sum<K>(wt, bias, win, u);
#pragma unroll
        for (int j = 0; j < V; ++j) {
          const float s = sigmoid(u[j]);
          g[j] *= s * __fmaf_rn(u[j], 1.f - s, 1.f);
        }
      }
      if (own) {
#pragma unroll
        for (int j = 0; j < V; ++j) {
          db[j] += g[j];
#pragma unroll
          for (int k = 0; k < K; ++k) dw[k][j] = __fmaf_rn(g[j], win[k][j], dw[k][j]);
        }
      }
#pragma unroll
      for (int b = 0; b < K; ++b)
#pragma unroll
        for (int j = 0; j < V; ++j) acc[b][j] = __fmaf_rn(wt[K - 1 - b][j], g[j], acc[b][j]);
    };
    const auto shift_sums = [&] {
#pragma unroll
      for (int j = 0; j < V; ++j) {
#pragma unroll
        for (int b = K - 1; b > 0; --b) acc[b][j] = acc[b - 1][j];
        acc[0][j] = 0.f;
      }
    };
    bool over = false;  // the chunk's last sequence has ended
    for (int at = t0; at < end && !over; at += R) {
      Strip<T, V> xn[R], gn[R];
#pragma unroll
      for (int i = 0; i < R; ++i) xn[i] = xv[i], gn[i] = gv[i];
      if (at + R < end) fetch(at + R);
      // the usual step: tokens of the chunk, whose sequence goes on behind them
      if (walk.end > at + R && at + R <= t1) {
        each<R>([&](auto step) {
          constexpr int i = decltype(step)::value;
          take(xn[i], gn[i], true);
          const int k = at + i, s = k - (K - 1);
          if (s >= max(t0, begin)) Strip<T, V>::store(dx + (int64_t)s * c.ld_dx, acc[K - 1], w.nv);
          else if (s < begin && begin >= t0 && c.dstate)
            Strip<T, V>::store(static_cast<T*>(c.dstate) + ((int64_t)walk.seq * (K - 1) + k - begin) * c.D + w.ch,
                               acc[K - 1], w.nv);
          shift_sums();
          conv_shift<K>(win);
        });
        continue;
      }
      each<R>([&](auto step) {
        constexpr int i = decltype(step)::value;
        const int k = at + i;
        if (k >= end || over) return;
        if (walk.next(c.seqs, k)) {
          if (k >= t1) {
            over = true;
            return;
          }
          begin = k;
          conv_window<T, K>(c, w, k, walk.seq, 0, win);
        }
        take(xn[i], gn[i], k < t1);
        // What is complete leaves: the input b tokens back, or that row of the state.
        const auto emit = [&](int b) {
          const int s = k - b;
          if (s >= begin) {
            if (s >= t0 && s < t1) Strip<T, V>::store(dx + (int64_t)s * c.ld_dx, acc[K - 1], w.nv);
          } else if (c.dstate && begin >= t0 && begin < t1) {
            Strip<T, V>::store(
                static_cast<T*>(c.dstate) + ((int64_t)walk.seq * (K - 1) + K - 1 + s - begin) * c.D + w.ch,
                acc[K - 1], w.nv);
          }
        };
        emit(K - 1);
        shift_sums();
        if (k + 1 == walk.end) {  // the others as well, with dlast's rows
#pragma unroll 1
          for (int b = K - 2; b >= 0; --b) {
            if (c.dlast) {
              float d[V];
              conv_state<T>(c, c.dlast, K, walk.seq, K - 2 - b, w, d);
#pragma unroll
              for (int j = 0; j < V; ++j) acc[K - 1][j] += d[j];
            }
            emit(b);
            shift_sums();
          }
        }
        conv_shift<K>(win);
      });
    }
  }

  // the workgroup's chunks, in order
#pragma unroll
  for (int k = 0; k <= K; ++k) {
    __syncthreads();
#pragma unroll
    for (int j = 0; j < V; j += 4) {
      const float* v = k < K ? dw[k < K ? k : 0] : db;
      st4(red + t * V + j, f4{v[j], v[j + 1], v[j + 2], v[j + 3]});
    }
    __syncthreads();
    for (int i = t; i < V * CT; i += kBlock) {
      const int ch = block * V * CT + i, first = ch - i % V;  // of the strip
      if (ch >= c.D) continue;
      const int at = i + (c.D >= V ? max(0, first + V - c.D) : 0);
      float v = 0.f;
      for (int j = 0; j < TL; ++j) v += red[j * V * CT + at];
      c.part[((int64_t)group * (K + 1) + k) * c.D + ch] = v;
    }
  }
}

// dw and the bias's gradient from the groups' sums: 16 of them to a workgroup, a sixteenth
// of the groups to each thread.
__global__ __launch_bounds__(kBlock) void k_convolution_sums(ConvCall c, int K) {
  const int64_t o = (int64_t)blockIdx.x * kSumOutputs + threadIdx.x % kSumOutputs, all = (int64_t)(K + 1) * c.D;
  const float v = sum_parts(c.part + o, all, c.groups, o < all);
  if (threadIdx.x >= kSumOutputs || o >= all) return;
  const int64_t k = o / c.D, ch = o % c.D;
  if (k < K) c.dweight[ch * K + k] = v;
  else if (c.dbias) c.dbias[ch] = v;
}

}  // namespace pg
