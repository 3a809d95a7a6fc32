// Gated linear recurrence over packed sequences, and its gradient: one scan
//   s <- a s + b
// over the tokens, for every channel on its own, with the state set anew where a
// sequence starts.  Forward s is h and b is x or (1 - a) x; the gradient runs
// against the reading direction with s = mu and b = a dh (lambda = dh + mu).
//
// The scan is cut along the tokens: a workgroup takes a chunk of L = rows * R
// tokens and a tile of channels.  A thread holds R consecutive tokens of four
// channels in registers and reduces them to one step (A, B): s_out = A s_in + B.
// The workgroup's rows of threads are joined through LDS, the chunks through
// words in memory: a chunk publishes its own (A, B) and, once it knows the state
// that enters it, the state that leaves it, so a later chunk looks back only as
// far as the nearest published state.  Every tensor is then read once and written
// once, and a long sequence is as parallel as many short ones.
//
// What a reset leaves behind is never multiplied by zero but dropped, so that
// infinities and NaN stay in their sequence.
#pragma once
#include "formats.h"
#include "operators.h"

namespace pg {

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
// The form of a gate that a thread keeps: the gate itself, or s with the gate's sign.
template <int FORM>
__device__ __forceinline__ float keep_gate(float g) {
  if constexpr (FORM == POLYGLOT_GATE_RAW) return g;
  return __builtin_copysignf(
      __builtin_amdgcn_exp2f(-0.72134752044448170f * __builtin_fabsf(g)), g);
}
template <int FORM>
__device__ __forceinline__ Decay decay(float kept) {
  if constexpr (FORM == POLYGLOT_GATE_RAW) return Decay{kept, 1.f, 1.f, 1.f};
  const float s = __builtin_fabsf(kept);
  const float r = __builtin_amdgcn_rcpf(1.f + s * s), q = s * r;
  return __float_as_int(kept) >= 0 ? Decay{r, q, q, s} : Decay{s * q, q, r, 1.f};
}

// The words that join the chunks.  Each is a value and a tag, written and read
// whole, so they need no order among themselves: a word counts once its tag is
// the launch's.  The first of a channel's two holds A; the second B, or with the
// tag's low bit set the state that leaves the chunk.
__device__ __forceinline__ void publish(uint64_t* w, float v, uint32_t tag) {
  __hip_atomic_store(w, (uint64_t)tag << 32 | __float_as_uint(v), __ATOMIC_RELAXED,
                     __HIP_MEMORY_SCOPE_AGENT);
}
__device__ __forceinline__ uint64_t observe(const uint64_t* w) {
  return __hip_atomic_load(w, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
}

__device__ __forceinline__ int64_t seq_offset(const RecCall& c, int i) {
  if (!c.offsets) return (int64_t)i * (c.tokens / c.nseq);
  return c.offset_bytes == 8 ? static_cast<const int64_t*>(c.offsets)[i]
                             : static_cast<const int32_t*>(c.offsets)[i];
}

// The first of the nseq + 1 offsets that is >= lo (nseq + 1 if none is), found by
// the whole wave: 64 probes split the range into 65 parts.
__device__ __forceinline__ int first_offset(const RecCall& c, int lo) {
  if (!c.offsets) {
    const int T = c.tokens / c.nseq;
    return T ? ceil_div(lo, T) : 0;
  }
  int l = 0, n = c.nseq + 1;  // the answer is in [l, l + n]
  while (n > 0) {
    const int step = ceil_div(n, kWave + 1);
    const int i = l + (lane_id() + 1) * step - 1;
    const bool below = i < l + n && seq_offset(c, i) < lo;
    const int k = __popcll(__ballot(below));  // of ascending offsets the first k are below
    l += k * step;
    n = min(step - 1, n - k * step);
  }
  return l;
}

// Tokens of a thread.
template <class T, bool GRAD>
constexpr int scan_tokens() {
  return sizeof(T) == 2 && !GRAD ? 16 : 8;
}

// LDS of a scan.
constexpr int kScanMinLanes = 8;                            // lanes of a row of threads
constexpr int kScanMaxRows = kBlock / kScanMinLanes;
constexpr int kScanMaxTokens = kScanMaxRows * 16;
struct ScanLds {
  int start[kScanMaxTokens];  // by place in the scan: the sequence that starts here, or -1
  int stop[kScanMaxTokens];   // ... that the scan ends here, or -1
  float a[4 * kBlock], b[4 * kBlock];  // steps of the rows of threads, [row][4][lanes]
  uint32_t done[kBlock];
  uint8_t cut[kScanMaxRows];  // a row of threads meets the start of a sequence
  int empty[kBlock];          // sequences without tokens
  int n_empty;
  uint64_t ticket;
};

constexpr int kScanLook = 2;                    // chunks that a row of threads looks back over
constexpr uint32_t kScanSpinLimit = 1u << 22;   // a wait that only a library bug makes

template <class T, int FORM, bool GRAD, bool SHARED, bool VEC, int R>
__global__ __launch_bounds__(kBlock) void k_scan(RecCall c, ScanPlan p) {
  __shared__ ScanLds s;
  const int t = threadIdx.x;
  const int CT = 1 << p.lanes_log2, TT = kBlock >> p.lanes_log2;
  const int cl = t & (CT - 1), tl = t >> p.lanes_log2, L = TT * R;

  // The chunks of a tile are handed out in the order in which workgroups start, so
  // every chunk that a look-back waits for is running or done.  Who takes the last
  // one makes the counter ready for the next launch.
  const int tile = blockIdx.x % p.tiles;
  int chunk = blockIdx.x / p.tiles;
  uint32_t tag = 0;
  if (p.head) {
    if (t == 0) {
      uint64_t* head = p.head + tile * kHeadLine;
      s.ticket = __hip_atomic_fetch_add(head, (uint64_t)1, __ATOMIC_RELAXED,
                                        __HIP_MEMORY_SCOPE_AGENT);
      if ((uint32_t)s.ticket == (uint32_t)p.chunks - 1) {
        const uint32_t next = (uint32_t)(s.ticket >> 32) + 1;
        __hip_atomic_store(head, (uint64_t)(next >> 31 ? 1u : next) << 32, __ATOMIC_RELAXED,
                           __HIP_MEMORY_SCOPE_AGENT);
      }
    }
    __syncthreads();
    chunk = (int)(uint32_t)s.ticket;
    tag = (uint32_t)(s.ticket >> 32) << 1;
  }

  // this thread's channels [ch, ch + nv) and their gate
  int ch, nv, gate_col = 0, part = 0;
  if constexpr (SHARED) {
    const int gi = cl / p.lanes_per_group, g = tile * p.groups_per_tile + gi;
    part = cl - gi * p.lanes_per_group;
    gate_col = g;
    ch = g * c.group + 4 * part;
    nv = gi < p.groups_per_tile && ch < c.D ? min(4, c.group - 4 * part) : 0;
  } else {
    ch = (tile * CT + cl) * 4;
    nv = max(0, min(4, c.D - ch));
  }
  const bool live = nv > 0;

  // tokens of the chunk: places [0, count) of the scan, token = t0 + place * dir
  const int q0 = chunk * L, count = min(L, c.tokens - q0);
  const int dir = c.down ? -1 : 1, t0 = c.down ? c.tokens - 1 - q0 : q0;
  const int lo = c.down ? t0 - count + 1 : t0, hi = lo + count;

  // every load of the chunk, in flight before anything waits (places past the end
  // and idle lanes load something that exists)
  Quad<T> in[R], hp[GRAD ? R : 1], xs[GRAD && FORM == POLYGLOT_GATE_SIGMOID ? R : 1];
  Quad<T> gq[SHARED ? 1 : R];
  T gs[SHARED ? R : 1];
  if (count > 0) {
    const int at = live ? ch : 0, col = live ? gate_col : 0;
#pragma unroll
    for (int i = 0; i < R; ++i) {
      const int place = min(tl * R + i, count - 1);
      const int64_t n = t0 + place * dir;
      if constexpr (SHARED) gs[i] = static_cast<const T*>(c.gate)[n * c.ld_gate + col];
      else gq[i] = load_quad<T, VEC>(static_cast<const T*>(c.gate) + n * c.ld_gate + at, nv);
      if constexpr (GRAD) {
        in[i] = load_quad<T, VEC>(static_cast<const T*>(c.dh) + n * c.ld_dh + at, nv);
        // the state before this token in reading order: the next one of this scan
        const int64_t m = q0 + place + 1 < c.tokens ? n + dir : n;
        hp[i] = load_quad<T, VEC>(static_cast<const T*>(c.h) + m * c.ld_h + at, nv);
        if constexpr (FORM == POLYGLOT_GATE_SIGMOID)
          xs[i] = load_quad<T, VEC>(static_cast<const T*>(c.x) + n * c.ld_x + at, nv);
      } else {
        in[i] = load_quad<T, VEC>(static_cast<const T*>(c.x) + n * c.ld_x + at, nv);
      }
    }
  }

  // where sequences start and stop in the chunk
  for (int i = t; i < L; i += kBlock) s.start[i] = s.stop[i] = -1;
  if (t == 0) s.n_empty = 0;
  const int n_off = c.nseq + 1;
  __syncthreads();
  for (int base = first_offset(c, lo); base < n_off; base += kBlock) {
    const int i = base + t;
    bool more = false;
    if (i < n_off) {
      const int64_t o = seq_offset(c, i);
      if (o >= lo && o <= hi) {
        more = true;
        if (i < c.nseq) {
          const int64_t next = seq_offset(c, i + 1);
          if (next > o && o < hi) {
            if (c.down) s.stop[hi - 1 - (int)o] = i;
            else s.start[(int)o - lo] = i;
          }
          if (next == o && (o < hi || hi == c.tokens)) s.empty[atomicAdd(&s.n_empty, 1)] = i;
        }
        if (i > 0 && o > lo && seq_offset(c, i - 1) < o) {
          if (c.down) s.start[hi - (int)o] = i - 1;
          else s.stop[(int)o - 1 - lo] = i - 1;
        }
      }
    }
    const bool again = __syncthreads_and(more);  // all 256 were in reach: there may be more
    if (c.fin && live)
      for (int k = tl; k < s.n_empty; k += TT)
        for (int v = 0; v < nv; ++v) {
          const size_t at = (size_t)s.empty[k] * c.D + ch + v;
          c.fin[at] = c.init ? c.init[at] : 0.f;
        }
    if (!again) break;
    __syncthreads();
    if (t == 0) s.n_empty = 0;
    __syncthreads();
  }
  // offsets that do not ascend from 0 to the tokens: each pair is looked at once
  if (c.offsets)
    for (int64_t i = (int64_t)blockIdx.x * kBlock + t; i <= c.nseq; i += (int64_t)gridDim.x * kBlock) {
      const int64_t o = seq_offset(c, (int)i);
      const int64_t next = i < c.nseq ? seq_offset(c, (int)i + 1) : c.tokens;
      if ((i == 0 && o != 0) || next < o || (i == c.nseq && o != c.tokens))
        atomicOr(c.flag, kFlagBadOffset);
    }

  // this thread's tokens as one step.  The state that a sequence starts with joins
  // what its first token adds, and is not read again: fin may be init.
  float a[R][SHARED ? 1 : 4];  // forward: decays; gradient: gates in the form that is kept
  float b[R][4];               // forward: what a token adds; gradient: dh
  float A[4], B[4];
  bool cut = false;
#pragma unroll
  for (int v = 0; v < 4; ++v) A[v] = 1.f, B[v] = 0.f;
#pragma unroll
  for (int i = 0; i < R; ++i) {
    const int place = tl * R + i;
    if (place >= count) break;
    const int from = s.start[place];
    float start[4] = {0.f, 0.f, 0.f, 0.f};
    if (from >= 0) {
      cut = true;
#pragma unroll
      for (int v = 0; v < 4; ++v) {
        B[v] = 0.f;
        if (v < nv && c.init) start[v] = c.init[(size_t)from * c.D + ch + v];
      }
    }
    Decay d{};
#pragma unroll
    for (int v = 0; v < 4; ++v) {
      if (!SHARED || v == 0) {
        const float kept = keep_gate<FORM>(SHARED ? Elem<T>::get(gs[SHARED ? i : 0])
                                                  : gq[SHARED ? 0 : i].get(v));
        d = decay<FORM>(kept);
        a[i][SHARED ? 0 : v] = GRAD ? kept : d.a;
      }
      if constexpr (GRAD) {
        b[i][v] = in[i].get(v) + start[v];
        B[v] = d.a * (b[i][v] + B[v]);
      } else {
        b[i][v] = d.rest(in[i].get(v));
        if (from >= 0) b[i][v] = __fmaf_rn(d.a, start[v], b[i][v]);
        B[v] = __fmaf_rn(d.a, B[v], b[i][v]);
      }
      A[v] *= d.a;
    }
  }
#pragma unroll
  for (int v = 0; v < 4; ++v) {
    s.a[(tl * 4 + v) * CT + cl] = A[v];
    s.b[(tl * 4 + v) * CT + cl] = B[v];
  }
  if (cl == 0) s.cut[tl] = cut;
  __syncthreads();

  // the step of the rows before this one, and for the last row that of the chunk
  float pa[4] = {1.f, 1.f, 1.f, 1.f}, pb[4] = {0.f, 0.f, 0.f, 0.f};
  bool pcut = false;
  for (int r = 0; r < tl; ++r) {
    const bool k = s.cut[r];
#pragma unroll
    for (int v = 0; v < 4; ++v) {
      const float ra = s.a[(r * 4 + v) * CT + cl], rb = s.b[(r * 4 + v) * CT + cl];
      pb[v] = k ? rb : __fmaf_rn(ra, pb[v], rb);
      pa[v] *= ra;
    }
    pcut |= k;
  }
  const bool ends = tl == TT - 1 && live && chunk + 1 < p.chunks;
  const bool set = chunk == 0 || pcut || cut;  // the chunk's end does not depend on its beginning
  uint64_t* const tile_words = p.words + tile * p.stride + cl;
  uint64_t* words = tile_words + (size_t)chunk * 8 * CT;  // [2][4][lanes]
  if (ends && p.head) {
#pragma unroll
    for (int v = 0; v < 4; ++v) {
      const float eb = cut ? B[v] : __fmaf_rn(A[v], pb[v], B[v]);
      if (set) {
        publish(words + (4 + v) * CT, eb, tag | 1u);
      } else {
        publish(words + v * CT, A[v] * pa[v], tag);
        publish(words + (4 + v) * CT, eb, tag);
      }
    }
  }

  // the state that enters the chunk
  float carry[4] = {0.f, 0.f, 0.f, 0.f};
  if (chunk > 0 && s.start[0] < 0 && p.head) {
    __syncthreads();  // the rows' steps are read
    float ca[4] = {1.f, 1.f, 1.f, 1.f};
    uint32_t found = live ? 0u : 15u;  // by channel: a published state was reached
    for (int base = chunk - 1;; base -= TT * kScanLook) {
      uint64_t wa[kScanLook][4], wb[kScanLook][4];
      uint32_t spins = 0;
      bool wait;
      do {
        wait = false;
#pragma unroll
        for (int k = 0; k < kScanLook; ++k) {
          const int j = base - tl * kScanLook - k;
          const uint64_t* w = tile_words + (int64_t)j * 8 * CT;
#pragma unroll
          for (int v = 0; v < 4; ++v) {
            // before the first chunk there is nothing: a state of 0 stands there
            wb[k][v] = (uint64_t)(tag | 1u) << 32;
            wa[k][v] = 0;
            if (live && j >= 0) {
              wb[k][v] = observe(w + (4 + v) * CT);
              wa[k][v] = observe(w + v * CT);
            }
          }
        }
#pragma unroll
        for (int k = 0; k < kScanLook; ++k)
#pragma unroll
          for (int v = 0; v < 4; ++v) {
            const uint32_t tb = (uint32_t)(wb[k][v] >> 32), ta = (uint32_t)(wa[k][v] >> 32);
            if (tb != (tag | 1u) && (tb != tag || ta != tag)) wait = true;
          }
        if (wait) {
          if (++spins > kScanSpinLimit) {
            atomicOr(c.flag, kFlagInternal);
            break;
          }
          __builtin_amdgcn_s_sleep(1);
        }
      } while (wait);
      // nearest first: this row's chunks as one step, or up to a state
      uint32_t mine = 0;
#pragma unroll
      for (int v = 0; v < 4; ++v) {
        float la = 1.f, lb = 0.f;
#pragma unroll
        for (int k = 0; k < kScanLook; ++k) {
          if (mine >> v & 1u) continue;
          lb = __fmaf_rn(la, __uint_as_float((uint32_t)wb[k][v]), lb);
          if ((uint32_t)(wb[k][v] >> 32) & 1u) mine |= 1u << v;
          else la *= __uint_as_float((uint32_t)wa[k][v]);
        }
        s.a[(tl * 4 + v) * CT + cl] = la;
        s.b[(tl * 4 + v) * CT + cl] = lb;
      }
      s.done[tl * CT + cl] = mine;
      __syncthreads();
      for (int r = 0; r < TT && found != 15u; ++r) {
        const uint32_t m = s.done[r * CT + cl];
#pragma unroll
        for (int v = 0; v < 4; ++v) {
          if (found >> v & 1u) continue;
          carry[v] = __fmaf_rn(ca[v], s.b[(r * 4 + v) * CT + cl], carry[v]);
          ca[v] *= s.a[(r * 4 + v) * CT + cl];
        }
        found |= m;
      }
      if (__syncthreads_and(found == 15u)) break;
    }
  }
  float st[4];
#pragma unroll
  for (int v = 0; v < 4; ++v) st[v] = pcut ? pb[v] : __fmaf_rn(pa[v], carry[v], pb[v]);
  if (ends && !set && p.head) {
#pragma unroll
    for (int v = 0; v < 4; ++v) publish(words + (4 + v) * CT, __fmaf_rn(A[v], st[v], B[v]), tag | 1u);
  }

  // the tokens again, now with the state before each
#pragma unroll
  for (int i = 0; i < R; ++i) {
    const int place = tl * R + i;
    if (place >= count) break;
    const int64_t n = t0 + place * dir;
    const int from = s.start[place], to = s.stop[place];
    if (from >= 0) st[0] = st[1] = st[2] = st[3] = 0.f;
    float o[4], dg[4];
    Decay d{};
#pragma unroll
    for (int v = 0; v < 4; ++v) {
      if constexpr (GRAD) {
        if (!SHARED || v == 0) d = decay<FORM>(a[i][SHARED ? 0 : v]);
        const float lam = b[i][v] + st[v];
        float h = hp[i].get(v);
        if (to >= 0) h = v < nv && c.h0 ? c.h0[(size_t)to * c.D + ch + v] : 0.f;
        o[v] = d.rest(lam);
        const float w = FORM == POLYGLOT_GATE_SIGMOID
                            ? lam * (h - xs[FORM == POLYGLOT_GATE_SIGMOID ? i : 0].get(v))
                            : lam * h;
        dg[v] = v < nv ? (SHARED ? w : d.slope(w)) : 0.f;
        st[v] = d.a * lam;
      } else {
        st[v] = __fmaf_rn(a[i][SHARED ? 0 : v], st[v], b[i][v]);
        o[v] = st[v];
      }
    }
    if (live) {
      store_quad<T, VEC>(static_cast<T*>(c.out) + n * c.ld_out + ch, o, nv);
      if (to >= 0 && c.fin)
        for (int v = 0; v < 4; ++v)
          if (v < nv) c.fin[(size_t)to * c.D + ch + v] = st[v];
    }
    if constexpr (GRAD && !SHARED) {
      if (live) store_quad<T, VEC>(static_cast<T*>(c.dgate) + n * c.ld_dgate + ch, dg, nv);
    } else if constexpr (GRAD) {
      // the group's lanes, in a fixed order: lane k holds the sum of [k, k + 2 o) after
      // the step of width o
      float sum = (dg[0] + dg[1]) + (dg[2] + dg[3]);
      for (int o = 1; o < p.lanes_per_group; o <<= 1) {
        const float other = __shfl_down(sum, o);
        if (part + o < p.lanes_per_group) sum += other;
      }
      if (live && part == 0)
        static_cast<T*>(c.dgate)[n * c.ld_dgate + gate_col] = Elem<T>::put(settled(d.slope(sum)));
    }
  }
}

// One token for every sequence: nothing to scan.
template <class T, int FORM, bool VEC>
__global__ __launch_bounds__(kBlock) void k_recurrence_step(RecCall c) {
  const int quads = (c.D + 3) / 4;
  const int64_t total = (int64_t)c.tokens * quads;
  for (int64_t i = (int64_t)blockIdx.x * kBlock + threadIdx.x; i < total;
       i += (int64_t)gridDim.x * kBlock) {
    const int64_t n = i / quads;
    const int ch = (int)(i - n * quads) * 4, nv = min(4, c.D - ch);
    const T* gate = static_cast<const T*>(c.gate) + n * c.ld_gate;
    const size_t at = (size_t)n * c.D + ch;
    const Quad<T> x = load_quad<T, VEC>(static_cast<const T*>(c.x) + n * c.ld_x + ch, nv);
    Quad<float> h{};
    if (c.init) h = load_quad<float, VEC>(c.init + at, nv);
    Quad<T> g{};
    if (c.group == 1) g = load_quad<T, VEC>(gate + ch, nv);
    float o[4];
#pragma unroll
    for (int v = 0; v < 4; ++v) {
      const float gv = c.group == 1 ? g.get(v) : v < nv ? Elem<T>::get(gate[(ch + v) / c.group]) : 0.f;
      const Decay d = decay<FORM>(keep_gate<FORM>(gv));
      o[v] = __fmaf_rn(d.a, h.get(v), d.rest(x.get(v)));
    }
    store_quad<T, VEC>(static_cast<T*>(c.out) + n * c.ld_out + ch, o, nv);
    if (c.fin) store_quad<float, VEC>(c.fin + at, o, nv);
  }
}

}  // namespace pg
