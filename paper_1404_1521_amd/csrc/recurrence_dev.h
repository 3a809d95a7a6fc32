// Gated linear recurrence over packed sequences, and its gradient: one scan
//   s <- a s + b
// over the tokens, for every channel on its own, with the state set anew where a
// sequence starts.  Forward s is h and b is x or (1 - a) x; the gradient runs
// against the reading direction with s = mu and b = a dh (lambda = dh + mu).
//
// The scan is cut along the tokens: a workgroup takes a chunk of L = rows * R
// tokens and a tile of channels.  A thread holds R consecutive tokens of four
// channels in registers and reduces them to one step (A, B): s_out = A s_in + B.
// The workgroup's rows of threads are joined through LDS, the chunks through words
// in memory: a chunk publishes its (A, B), the last one of a group that of the group
// and, once it knows it, the state that leaves the group.  A chunk so reads the steps
// of at most 15 chunks and of the groups since the nearest known state.  Every tensor is then read once and written
// once, and a long sequence is as parallel as many short ones.
// What waits polls one word per chunk, which says what the chunk has published:
// polling the channels' own words took half of the memory's rate from the tensors.
//
// What a reset leaves behind is never multiplied by zero but dropped, so that
// infinities and NaN stay in their sequence.
//
// What bounds it.  Wide layers: memory, and the latency that two workgroups to a CU do
// not cover (224 registers; a forward wave waits 44% of its cycles, its vector
// instructions take 22%, 23 of them an element).  65,536 tokens 2,048 wide, bfloat16, 16
// documents: forward 231 us (3.5 TB/s of the tensors' 806 MB), gradient 420 us (3.8 TB/s
// of 1.61 GB); at the 5.17 TB/s of a large copy they take 156 and 312.  Small calls: a
// chain of dependent rounds, 5.3 us in a workgroup alone: the ticket and the offsets 0.9,
// the loads' issue 0.6, the marks 1.2, the first pass 0.8, the join 0.8, the second pass
// 0.7; 2.4 more where chunks wait for each other.  16,384 x 128 float32 in 700 sentences
// forward 14.7 us, 16,411 x 256 bfloat16 with 8 gates gradient 21.7 us, one sequence of
// 65,537 x 64 float32 gradient 28 us (at a copy's rate 4.9, 6.6, 16.2).
#pragma once
#include <type_traits>

#include "formats.h"
#include "operators.h"

namespace pg {

// What a gate does: the decay a, and for a gate before its sigmoid the products
// with 1 - a and with the sigmoid's slope a (1 - a).  With s = e^(-|gate| / 2),
// r = 1 / (1 + s^2) and q = s r, the larger one of a and 1 - a is r, the other s q,
// and the slope q^2: nothing is lost to a subtraction, and a product taken factor
// by factor keeps its digits where 1 - a alone is below the normal floats.  The
// hardware's base-2 exponential and reciprocal are good to one unit in the last place;
// the exponential's argument is a rounded product, so that s^2 is off by about |gate|
// half units more.
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

// The decay and 1 - a of the forward pass, where a product with either is a share of a
// larger sum: r = 1 / (1 + e^-gate), and 1 - r, or where r is above a half e^-gate r.
template <int FORM>
__device__ __forceinline__ void gate_pair(float g, float& a, float& rest) {
  if constexpr (FORM == POLYGLOT_GATE_RAW) {
    a = g;
    rest = 1.f;
  } else {
    const float e = __builtin_amdgcn_exp2f(-1.44269504088896341f * g);
    a = __builtin_amdgcn_rcpf(1.f + e);
    rest = a > 0.5f ? e * a : 1.f - a;
  }
}

// The words that join the chunks.  Each is a value and a tag, written and read
// whole, so they need no order among themselves: a word counts once its tag is the
// launch's.  A channel has two for a chunk, its step (A, B), and three for a group of
// chunks: its step, and the state that leaves it.  A flag tells what a chunk or a group
// has out: its step; or its end, known without its beginning (a chunk's B, a group's
// state).
constexpr uint32_t kPartStep = 1, kPartEnd = 2;
__device__ __forceinline__ void publish(uint64_t* w, uint32_t v, uint32_t tag) {
  __hip_atomic_store(w, (uint64_t)tag << 32 | v, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
}
__device__ __forceinline__ uint64_t observe(const uint64_t* w) {
  return __hip_atomic_load(w, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
}

constexpr uint32_t kScanSpinLimit = 1u << 22;  // a wait that only a library bug makes

// A tile's flags and words.
struct ScanTile {
  uint64_t *chunk_flags, *group_flags, *words;
  uint32_t tag;
  int chunks, lanes;
  __device__ __forceinline__ ScanTile(const ScanPlan& p, int tile, uint32_t tag)
      : tag(tag), chunks(p.chunks), lanes(1 << p.lanes_log2) {
    const int groups = (p.chunks >> p.group_log2) + 1;
    chunk_flags = p.flags + (size_t)tile * (p.chunks + groups);
    group_flags = chunk_flags + p.chunks;
    words = p.words + (size_t)tile * (8 * (size_t)p.chunks + 12 * (size_t)groups) * lanes;
  }
  __device__ __forceinline__ uint64_t* step(int chunk) const {  // [2][4][lanes]
    return words + (size_t)chunk * 8 * lanes;
  }
  __device__ __forceinline__ uint64_t* group_step(int group) const {  // [3][4][lanes]
    return words + ((size_t)chunks * 8 + (size_t)group * 12) * lanes;
  }
  // Values that a flag has announced: a from row `ra` of w on (1 if ra < 0), b from row rb.
  __device__ __forceinline__ void read(const uint64_t* w, int CT, int ra, int rb, float (&a)[4],
                                       float (&b)[4], uint32_t* error) const {
    for (uint32_t spins = 0;; ++spins) {
      bool wait = false;
      uint64_t wa[4], wb[4];
#pragma unroll
      for (int v = 0; v < 4; ++v) {
        wa[v] = (uint64_t)tag << 32 | 0x3f800000u;
        if (ra >= 0) wa[v] = observe(w + (ra + v) * CT);
        wb[v] = observe(w + (rb + v) * CT);
      }
#pragma unroll
      for (int v = 0; v < 4; ++v) {
        wait |= (uint32_t)(wa[v] >> 32) != tag || (uint32_t)(wb[v] >> 32) != tag;
        a[v] = __uint_as_float((uint32_t)wa[v]);
        b[v] = __uint_as_float((uint32_t)wb[v]);
      }
      if (!wait) return;
      if (spins > kScanSpinLimit) {
        atomicOr(error, kFlagInternal);
        return;
      }
    }
  }
};

// Offset i; what no count of tokens can be raises the flag and is taken as the
// nearest one.
__device__ __forceinline__ int seq_offset(const RecCall& c, int i) {
  if (!c.offsets) return i * (c.tokens / c.nseq);
  if (c.offset_bytes == 4) return static_cast<const int32_t*>(c.offsets)[i];
  const int64_t o = static_cast<const int64_t*>(c.offsets)[i];
  if (o < 0 || o > INT32_MAX) atomicOr(c.flag, kFlagBadOffset);
  return (int)min(max(o, (int64_t)0), (int64_t)INT32_MAX);
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
    n -= k * step;
    if (k < kWave) n = min(step - 1, n);  // the next probe is not below
  }
  return l;
}

// Tokens of a thread.  More of them are fewer chunks and fewer joining words, and more
// registers: two workgroups of 256 threads to a CU, and no vectors spilled.  65,536 tokens
// 2,048 wide, one sequence, us.  Forward: bfloat16 sigmoid 12 tokens 278, 16 246; raw 12
// 262, 16 233; float32 raw 12 362, 16 328; sigmoid 8 (three workgroups to a CU) 367, 12
// 374, 16 (spilling) 451: 8 and 12 are as good as each other, 25.8 and 25.7 at 65,537 x 64,
// 33 and 32 to 35 at 16,384 x 512.  Gradient: bfloat16 sigmoid 8 490, 10 465, 12 428; raw 8
// 360, 10 385, 12 353; float32 sigmoid 8 659, 10 (spilling) 715; raw 8 572, 10 542, which
// the sigmoid decides for both.
template <class T, int FORM, bool GRAD>
constexpr int scan_tokens() {
  if (sizeof(T) == 2) return GRAD ? 12 : 16;
  return GRAD ? 8 : FORM == POLYGLOT_GATE_RAW ? 16 : 12;
}
constexpr int kScanMinTokens = 8;
// ... and of calls that so have fewer workgroups than there are CUs: their time
// is latency, and a thread's share of the work is part of it: 172 workgroups of 12 tokens
// a thread (16,384 x 128 float32 forward) 16.6 us, with 4 tokens 14.6; but 344 of 12
// (16,411 x 256 bfloat16, shared gates' gradient) 21.7, with 4 25.1.
constexpr int kScanShortTokens = 4;
constexpr int kScanFewWorkgroups = kCus;
constexpr int kScanMinLanes = 8;  // of a row of threads

// A value of another lane of the row of 16: quad_perm 0xb1 and 0x4e (the neighbour, the
// other pair), 0x141 the half mirrored, 0x140 the row mirrored.
template <int CTRL>
__device__ __forceinline__ float dpp_moved(float v) {
  return __int_as_float(__builtin_amdgcn_update_dpp(0, __float_as_int(v), CTRL, 0xf, 0xf, true));
}

// LDS of a scan.
constexpr int kLookEnd = 256;     // ScanLds::look: an end lies before the steps
constexpr int kScanMaxMates = 16; // chunks of a group
constexpr int kScanBatch = 1024;               // offsets read at a time
constexpr int kScanMateSlots = 16 * 4 * 32;  // 16 chunks of 32 lanes or 8 of 64
template <int R>
struct ScanLds {
  static constexpr int kTokens = kBlock / kScanMinLanes * R;  // most of a chunk
  int start[kTokens];  // by place in the scan: the sequence that starts here, or -1
  int stop[kTokens];   // ... that the scan ends here, or -1
  float a[4 * kBlock], b[4 * kBlock];    // steps of the waves, [wave][4][lanes]
  float ea[4 * kWave], eb[4 * kWave];  // the chunk's step
  float la[4 * kBlock], lb[4 * kBlock];        // steps of the groups before, [row][4][lanes]
  float ma[kScanMateSlots], mb[kScanMateSlots];  // ... of the group's chunks before, [chunk][4][lanes]
  int off[kScanBatch + 2];       // a batch of offsets, from the one before it on
  uint8_t cut[kWavesPerBlock];       // a wave meets the start of a sequence
  int empty[kScanBatch];         // sequences without tokens
  int n_empty;
  int any;                       // a sequence starts or stops in the chunk
  int look;                      // steps to take
  uint64_t ticket;
};

template <class T, int FORM, bool GRAD, bool SHARED, bool VEC, int R>
__global__ __launch_bounds__(kBlock, 2) void k_scan(RecCall c, ScanPlan p) {
  constexpr bool kUsesX = GRAD && FORM == POLYGLOT_GATE_SIGMOID;
  __shared__ ScanLds<R> s;
  const int t = threadIdx.x;
  const int CT = 1 << p.lanes_log2, TT = kBlock >> p.lanes_log2;
  const int cl = t & (CT - 1), tl = t >> p.lanes_log2, L = TT * R;
  const int tile = blockIdx.x % p.tiles;

  // The chunks of a tile are handed out in the order in which workgroups start, so
  // every chunk that a look-back waits for is running or done.
  uint64_t ticket = blockIdx.x / p.tiles;
  if (t == 0 && p.head)
    ticket = __hip_atomic_fetch_add(p.head + tile * kHeadLine, (uint64_t)1, __ATOMIC_RELAXED,
                                    __HIP_MEMORY_SCOPE_AGENT);

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
  const int own = live ? ch : 0, col = live ? gate_col : 0;  // idle lanes load something that exists

  // Offsets, a batch at a time with the neighbours of its ends, asked for at once.
  // Where that is all of them they are read while the ticket is on its way; otherwise
  // those near the chunk are searched for.
  const int n_off = c.nseq + 1;
  const bool all = n_off <= kScanBatch;
  const auto load_offsets = [&](int base) {
    constexpr int kEach = (kScanBatch + 2 + kBlock - 1) / kBlock;
    int o[kEach];
#pragma unroll
    for (int j = 0; j < kEach; ++j)
      o[j] = base + j * kBlock + t <= n_off ? seq_offset(c, max(base + j * kBlock + t - 1, 0)) : 0;
#pragma unroll
    for (int j = 0; j < kEach; ++j)
      if (j * kBlock + t < kScanBatch + 2) s.off[j * kBlock + t] = o[j];
  };
  if (all) load_offsets(0);
  for (int i = t; i < L; i += kBlock) s.start[i] = s.stop[i] = -1;
  if (t == 0) {
    s.n_empty = s.any = 0;
    s.ticket = ticket;
  }
  __syncthreads();
  const uint32_t tag = (uint32_t)(s.ticket >> 32);
  const int chunk = (int)(uint32_t)s.ticket;
  // A ticket past the chunks: another call, which the program lets overlap with this one,
  // draws from the same counter.  Its place would lie outside of the tile's words.
  if ((uint32_t)chunk >= (uint32_t)p.chunks) {
    if (t == 0) atomicOr(c.flag, kFlagInternal);
    return;
  }

  // The chunk's tokens are the places [0, count) of the scan from q0 on: token
  // t0 + place * dir.
  const int q0 = chunk * L, count = min(L, c.tokens - q0);
  const int dir = c.down ? -1 : 1, t0 = c.down ? c.tokens - 1 - q0 : q0;
  const int lo = c.down ? t0 - count + 1 : t0, hi = lo + count;

  // Every load of the chunk, in flight before anything waits: the thread's tokens, and
  // of a gradient the states before them in reading order, the next ones of this scan.
  // Places past the end load the last one.
  Quad<T> in[R], gq[SHARED ? 1 : R], hp[GRAD ? R : 1], xs[kUsesX ? R : 1];
  T gs[SHARED ? R : 1];
  const int64_t first = t0 + (int64_t)tl * R * dir;  // the thread's first token
  if (count > 0) {
    const T* gate = static_cast<const T*>(c.gate) + first * c.ld_gate + (SHARED ? col : own);
    const T* step = static_cast<const T*>(GRAD ? c.dh : c.x) + first * (GRAD ? c.ld_dh : c.ld_x) + own;
    const T* h = GRAD ? static_cast<const T*>(c.h) + (first + dir) * c.ld_h + own : nullptr;
    const T* x = kUsesX ? static_cast<const T*>(c.x) + first * c.ld_x + own : nullptr;
    const int64_t gate_ld = dir * c.ld_gate, step_ld = dir * (GRAD ? c.ld_dh : c.ld_x);
    const int64_t h_ld = dir * c.ld_h, x_ld = dir * c.ld_x;
    const auto load = [&](int i, int k, int kh) {
      if constexpr (SHARED) gs[i] = gate[k * gate_ld];
      else gq[i] = load_quad<T, VEC>(gate + k * gate_ld, nv);
      in[i] = load_quad<T, VEC>(step + k * step_ld, nv);
      if constexpr (GRAD) hp[i] = load_quad<T, VEC>(h + kh * h_ld, nv);
      if constexpr (kUsesX) xs[i] = load_quad<T, VEC>(x + k * x_ld, nv);
    };
    if (q0 + (int64_t)L < c.tokens) {  // the chunk and the place after it are whole
#pragma unroll
      for (int i = 0; i < R; ++i) load(i, i, i);
    } else {
      const int last = count - 1 - tl * R, end = c.tokens - 1 - q0 - tl * R;
#pragma unroll
      for (int i = 0; i < R; ++i) load(i, min(i, last), min(min(i, last), end - 1));
    }
  }

  // where sequences start and stop in the chunk
  int base = 0;
  if (!all) {
    base = first_offset(c, lo);
    load_offsets(base);
    __syncthreads();
  }
  while (base < n_off) {
    bool more = false;
    for (int j = t; j < kScanBatch && base + j < n_off; j += kBlock) {
      const int i = base + j, o = s.off[j + 1];
      more = o >= lo && o <= hi;
      if (!more) continue;
      if (i < c.nseq) {
        const int after = s.off[j + 2];
        if (after > o && o < hi) {
          if (c.down) s.stop[hi - 1 - o] = i;
          else s.start[o - lo] = i;
          s.any = 1;
        }
        if (after == o && (o < hi || hi == c.tokens)) s.empty[atomicAdd(&s.n_empty, 1)] = i;
      }
      if (i > 0 && o > lo && s.off[j] < o) {
        if (c.down) s.start[hi - o] = i - 1;
        else s.stop[o - 1 - lo] = i - 1;
        s.any = 1;
      }
    }
    const bool again = __syncthreads_and(more);  // the batch's last ones were all in reach
    if (c.fin && live)
      for (int k = tl; k < s.n_empty; k += TT) {
        const size_t place = (size_t)s.empty[k] * c.D + ch;
        Quad<float> q{};
        if (c.init) q = load_quad<float, VEC>(c.init + place, nv);
        const float v[4] = {q.get(0), q.get(1), q.get(2), q.get(3)};
        store_quad<float, VEC>(c.fin + place, v, nv);
      }
    base += kScanBatch;
    if (!again || base >= n_off) break;
    load_offsets(base);
    __syncthreads();
    if (t == 0) s.n_empty = 0;
    __syncthreads();
  }

  // this thread's tokens as one step.  The state that a sequence starts with joins
  // what its first token adds, and is not read again: fin may be init.
  const bool any = s.any;
  float a[R][SHARED ? 1 : 4];  // forward: decays; gradient: gates in the form that is kept
  float b[R][4];               // forward: what a token adds; gradient: dh
  float A[4], B[4];
  bool cut = false;
#pragma unroll
  for (int v = 0; v < 4; ++v) A[v] = 1.f, B[v] = 0.f;
  // A chunk in the middle of a sequence has no ends and no missing tokens: it goes
  // through without a look at either (a branch for each token kept 7 moves per element).
  const bool plain = !any && count == L;
  const auto first_pass = [&](auto is_plain) {
    constexpr bool PLAIN = decltype(is_plain)::value;
#pragma unroll
    for (int i = 0; i < R; ++i) {
      float da[4], rest = 1.f;
#pragma unroll
      for (int v = 0; v < 4; ++v) {
        if (!SHARED || v == 0) {
          const float g = SHARED ? Elem<T>::get(gs[SHARED ? i : 0]) : gq[SHARED ? 0 : i].get(v);
          if constexpr (GRAD) {
            a[i][SHARED ? 0 : v] = keep_gate<FORM>(g);
            da[v] = decay<FORM>(a[i][SHARED ? 0 : v]).a;
          } else {
            gate_pair<FORM>(g, da[v], rest);
            a[i][SHARED ? 0 : v] = da[v];
          }
        } else {
          da[v] = da[0];
        }
        b[i][v] = in[i].get(v);
        if (!GRAD) b[i][v] *= rest;
      }
      if constexpr (!PLAIN) {
        const int from = s.start[tl * R + i];
        if (from >= 0) {
          cut = true;
          Quad<float> start{};
          if (c.init) start = load_quad<float, VEC>(c.init + (size_t)from * c.D + own, nv);
#pragma unroll
          for (int v = 0; v < 4; ++v) {
            B[v] = 0.f;
            b[i][v] = __fmaf_rn(GRAD ? 1.f : da[v], start.get(v), b[i][v]);
          }
        }
      }
      if (PLAIN || tl * R + i < count) {
#pragma unroll
        for (int v = 0; v < 4; ++v) {
          B[v] = GRAD ? da[v] * (b[i][v] + B[v]) : __fmaf_rn(da[v], B[v], b[i][v]);
          A[v] *= da[v];
        }
      }
    }
  };
  if (plain) first_pass(std::true_type{});
  else first_pass(std::false_type{});
  // The rows of a wave by doubling: [A, B] of the rows up to this one, closed where a
  // sequence starts in them (then A says nothing).  The waves through LDS.
  const int wave = t / kWave, lane = t & (kWave - 1);
  const bool head_row = lane < CT, last_row = lane >= kWave - CT;  // of the wave
  bool closed = cut;
  for (int o = CT; o < kWave; o <<= 1) {
    const bool uc = __shfl_up((int)closed, o);
#pragma unroll
    for (int v = 0; v < 4; ++v) {
      const float ua = __shfl_up(A[v], o), ub = __shfl_up(B[v], o);
      if (lane >= o) {
        if (!closed) B[v] = __fmaf_rn(A[v], ub, B[v]);
        A[v] *= ua;
      }
    }
    if (lane >= o) closed |= uc;
  }
  if (last_row) {
#pragma unroll
    for (int v = 0; v < 4; ++v) {
      s.a[(wave * 4 + v) * CT + cl] = A[v];
      s.b[(wave * 4 + v) * CT + cl] = B[v];
    }
    if (cl == 0) s.cut[wave] = closed;
  }
  __syncthreads();
  // the step of the waves before this one
  float pa[4] = {1.f, 1.f, 1.f, 1.f}, pb[4] = {0.f, 0.f, 0.f, 0.f};
  bool pcut = false;
  for (int r = 0; r < wave; ++r) {
    const bool k = s.cut[r];
#pragma unroll
    for (int v = 0; v < 4; ++v) {
      const float ra = s.a[(r * 4 + v) * CT + cl], rb = s.b[(r * 4 + v) * CT + cl];
      pb[v] = k ? rb : __fmaf_rn(ra, pb[v], rb);
      pa[v] *= ra;
    }
    pcut |= k;
  }
  // the last row has the chunk's step, or where a sequence starts in it, its end
  const bool ends = tl == TT - 1 && chunk + 1 < p.chunks && p.head;
  const bool set = chunk == 0 || pcut || closed;
  const ScanTile at(p, tile, tag);
  if (ends) {
#pragma unroll
    for (int v = 0; v < 4; ++v) {
      const float ea = A[v] * pa[v], eb = closed ? B[v] : __fmaf_rn(A[v], pb[v], B[v]);
      if (!set) publish(at.step(chunk) + v * CT + cl, __float_as_uint(ea), tag);
      publish(at.step(chunk) + (4 + v) * CT + cl, __float_as_uint(eb), tag);
      s.ea[v * CT + cl] = ea;
      s.eb[v * CT + cl] = eb;
    }
    if (cl == 0) publish(at.chunk_flags + chunk, set ? kPartEnd : kPartStep, tag);
  }
  // the step of all rows before this one
  {
    const bool uc = __shfl_up((int)closed, CT);
#pragma unroll
    for (int v = 0; v < 4; ++v) {
      const float ua = __shfl_up(A[v], CT), ub = __shfl_up(B[v], CT);
      if (!head_row) {
        pb[v] = uc ? ub : __fmaf_rn(ua, pb[v], ub);
        pa[v] *= ua;
      }
    }
    if (!head_row) pcut |= uc;
  }

  // The state that enters the chunk: that of its group's beginning, taken through the
  // steps of the group's chunks before it, one by one.  The group's beginning, likewise,
  // is the nearest group's end that is known, taken through the steps of the groups
  // after it.  What is summed in which order does not depend on who is how far.
  float carry[4] = {0.f, 0.f, 0.f, 0.f};
  const int G = 1 << p.group_log2, group = chunk >> p.group_log2, mates = chunk & (G - 1);
  const bool last_mate = mates == G - 1 && chunk + 1 < p.chunks;
  if (p.head && chunk > 0 && (s.start[0] < 0 || last_mate)) {
    uint64_t f = 0;
    if (t < kWave) {
      // lanes below 16: chunks of the group, the others: groups; nearest first
      const bool is_mate = t < kScanMaxMates;
      const int j = is_mate ? chunk - 1 - t : group - 1 - (t - kScanMaxMates);
      const bool there = is_mate ? t < mates : j >= 0;
      const uint64_t* const flag = (is_mate ? at.chunk_flags : at.group_flags) + (there ? j : 0);
      for (uint32_t spins = 0;; ++spins) {
        f = there ? observe(flag) : 0;
        const uint32_t what = there && (uint32_t)(f >> 32) == tag ? (uint32_t)f : 0u;
        f = what;
        const uint32_t out = (uint32_t)__ballot(is_mate && what != 0);
        const uint32_t end = (uint32_t)__ballot(is_mate && what == kPartEnd);
        const int n = end ? __builtin_ctz(end) : mates;  // steps to take
        const uint32_t nearer = (1u << n) - 1;
        if ((out & nearer) == nearer || spins > kScanSpinLimit) {
          if (spins > kScanSpinLimit) atomicOr(c.flag, kFlagInternal);
          if (t == 0) s.look = n | (end ? kLookEnd : 0);
          break;
        }
        __builtin_amdgcn_s_sleep(1);
      }
    }
    __syncthreads();
    const int n = s.look & (kLookEnd - 1);
    const bool end = s.look & kLookEnd;
    // [0, n): the steps, farthest first; n: the end before them
    for (int m = tl; m < n + (end ? 1 : 0); m += TT) {
      float va[4], vb[4];
      at.read(at.step(m < n ? chunk - n + m : chunk - 1 - n) + cl, CT, m < n ? 0 : -1, 4, va, vb, c.flag);
#pragma unroll
      for (int v = 0; v < 4; ++v) {
        s.ma[(m * 4 + v) * CT + cl] = va[v];
        s.mb[(m * 4 + v) * CT + cl] = vb[v];
      }
    }
    __syncthreads();
    // the group's own step, or its end
    const bool group_ends = last_mate && tl == TT - 1;
    const bool group_set = end || set;
    float ga[4], gb[4];
    if (group_ends) {
#pragma unroll
      for (int v = 0; v < 4; ++v) {
        ga[v] = 1.f;
        gb[v] = end ? s.mb[(n * 4 + v) * CT + cl] : 0.f;
      }
      for (int m = 0; m < n; ++m)
#pragma unroll
        for (int v = 0; v < 4; ++v) {
          const float a1 = s.ma[(m * 4 + v) * CT + cl];
          gb[v] = __fmaf_rn(a1, gb[v], s.mb[(m * 4 + v) * CT + cl]);
          ga[v] *= a1;
        }
#pragma unroll
      for (int v = 0; v < 4; ++v) {
        const float ea = s.ea[v * CT + cl], eb = s.eb[v * CT + cl];
        gb[v] = set ? eb : __fmaf_rn(ea, gb[v], eb);
        ga[v] *= ea;
        if (!group_set) {
          publish(at.group_step(group) + v * CT + cl, __float_as_uint(ga[v]), tag);
          publish(at.group_step(group) + (4 + v) * CT + cl, __float_as_uint(gb[v]), tag);
        } else {
          publish(at.group_step(group) + (8 + v) * CT + cl, __float_as_uint(gb[v]), tag);
        }
      }
      if (cl == 0) publish(at.group_flags + group, group_set ? kPartEnd : kPartStep, tag);
    }
    if (end) {
#pragma unroll
      for (int v = 0; v < 4; ++v) carry[v] = s.mb[(n * 4 + v) * CT + cl];
    } else if (group > 0 && (s.start[0] < 0 || !group_set)) {
      if (t < kWave) {
        const int j = group - 1 - (t - kScanMaxMates);
        const bool there = t >= kScanMaxMates && j >= 0;
        for (uint32_t spins = 0;; ++spins) {
          const uint64_t out = __ballot(there && f != 0) >> kScanMaxMates;
          const uint64_t state = __ballot(there && f == kPartEnd) >> kScanMaxMates;
          const int d = state ? __builtin_ctzll(state) : 0;
          const uint64_t nearer = ((uint64_t)1 << d) - 1;
          if ((state && (out & nearer) == nearer) || spins > kScanSpinLimit) {
            if (spins > kScanSpinLimit) atomicOr(c.flag, kFlagInternal);
            if (t == 0) s.look = min(d, group - 1);
            break;
          }
          __builtin_amdgcn_s_sleep(1);
          f = there ? observe(at.group_flags + j) : 0;
          f = (uint32_t)(f >> 32) == tag ? (uint32_t)f : 0u;
        }
      }
      __syncthreads();
      const int d = s.look;
      for (int m0 = 0; m0 <= d; m0 += TT) {
        if (m0 > 0) __syncthreads();
        const int m = m0 + tl;  // 0: the end; then the steps, nearer with m
        if (m <= d) {
          float va[4], vb[4];
          at.read(at.group_step(group - 1 - d + m) + cl, CT, m > 0 ? 0 : -1, m > 0 ? 4 : 8, va, vb, c.flag);
#pragma unroll
          for (int v = 0; v < 4; ++v) {
            s.la[(tl * 4 + v) * CT + cl] = va[v];
            s.lb[(tl * 4 + v) * CT + cl] = vb[v];
          }
        }
        __syncthreads();
        for (int r = 0; r < TT && m0 + r <= d; ++r)
#pragma unroll
          for (int v = 0; v < 4; ++v) {
            const float lb = s.lb[(r * 4 + v) * CT + cl];
            carry[v] = m0 + r == 0 ? lb : __fmaf_rn(s.la[(r * 4 + v) * CT + cl], carry[v], lb);
          }
      }
    }
    if (group_ends && !group_set) {
#pragma unroll
      for (int v = 0; v < 4; ++v)
        publish(at.group_step(group) + (8 + v) * CT + cl,
                __float_as_uint(__fmaf_rn(ga[v], carry[v], gb[v])), tag);
      if (cl == 0) publish(at.group_flags + group, kPartEnd, tag);
    }
    for (int m = 0; m < n; ++m)
#pragma unroll
      for (int v = 0; v < 4; ++v)
        carry[v] = __fmaf_rn(s.ma[(m * 4 + v) * CT + cl], carry[v], s.mb[(m * 4 + v) * CT + cl]);
  }
  float st[4];
#pragma unroll
  for (int v = 0; v < 4; ++v) st[v] = pcut ? pb[v] : __fmaf_rn(pa[v], carry[v], pb[v]);

  // the tokens again, now with the state before each
  T* out = static_cast<T*>(c.out) + first * c.ld_out + own;
  T* dgate = nullptr;
  if (GRAD)
    dgate = static_cast<T*>(c.dgate) + first * c.ld_dgate + (SHARED ? col : own);
  float sum[GRAD && SHARED ? R : 1];
  const auto second_pass = [&](auto is_plain) {
    constexpr bool PLAIN = decltype(is_plain)::value;
#pragma unroll
    for (int i = 0; i < R; ++i) {
      const bool ok = live && (PLAIN || tl * R + i < count);
      int to = -1;
      if constexpr (!PLAIN) {
        if (s.start[tl * R + i] >= 0) st[0] = st[1] = st[2] = st[3] = 0.f;
        to = s.stop[tl * R + i];
      }
      Quad<float> h0{};
      if (!PLAIN && GRAD && to >= 0 && c.h0) h0 = load_quad<float, VEC>(c.h0 + (size_t)to * c.D + own, nv);
      float o[4], dg[4];
      Decay d{};
#pragma unroll
      for (int v = 0; v < 4; ++v) {
        if constexpr (GRAD) {
          // (settled: computed again and not kept from the first pass)
          if (!SHARED || v == 0) d = decay<FORM>(settled(a[i][SHARED ? 0 : v]));
          const float lam = b[i][v] + st[v];
          float h = hp[i].get(v);
          if (!PLAIN && to >= 0) h = h0.get(v);
          o[v] = d.rest(lam);
          const float w = kUsesX ? lam * (h - xs[kUsesX ? i : 0].get(v)) : lam * h;
          dg[v] = SHARED ? (v < nv ? w : 0.f) : d.slope(w);
          st[v] = d.a * lam;
        } else {
          st[v] = __fmaf_rn(a[i][SHARED ? 0 : v], st[v], b[i][v]);
          o[v] = st[v];
        }
      }
      if (ok) {
        store_quad<T, VEC>(out, o, nv);
        if (!PLAIN && to >= 0 && c.fin) store_quad<float, VEC>(c.fin + (size_t)to * c.D + own, st, nv);
        if constexpr (GRAD && !SHARED) store_quad<T, VEC>(dgate, dg, nv);
      }
      if constexpr (GRAD && SHARED) sum[i] = (dg[0] + dg[1]) + (dg[2] + dg[3]);
      out += dir * c.ld_out;
      if (GRAD && !SHARED) dgate += dir * c.ld_dgate;
    }
  };
  if (plain) second_pass(std::true_type{});
  else second_pass(std::false_type{});
  if constexpr (GRAD && SHARED) {
    // The group's lanes, in a fixed order.  Powers of two by exchanges inside rows of 16
    // lanes (of neighbours, of pairs, halves mirrored, rows mirrored), then of rows;
    // other counts by doubling, lane k holding the sum of [k, k + 2 o) after the step of
    // width o.
    const int lanes = p.lanes_per_group;
    if ((lanes & (lanes - 1)) == 0) {
#pragma unroll
      for (int i = 0; i < R; ++i) {
        if (lanes > 1) sum[i] += dpp_moved<0xb1>(sum[i]);
        if (lanes > 2) sum[i] += dpp_moved<0x4e>(sum[i]);
        if (lanes > 4) sum[i] += dpp_moved<0x141>(sum[i]);
        if (lanes > 8) sum[i] += dpp_moved<0x140>(sum[i]);
        if (lanes > 16) sum[i] += __shfl_xor(sum[i], 16);
        if (lanes > 32) sum[i] += __shfl_xor(sum[i], 32);
      }
    } else {
      for (int o = 1; o < lanes; o <<= 1)
#pragma unroll
        for (int i = 0; i < R; ++i) {
          const float other = __shfl_down(sum[i], o);
          if (part + o < lanes) sum[i] += other;
        }
    }
    if (live && part == 0)
#pragma unroll
      for (int i = 0; i < R; ++i)
        if (tl * R + i < count)
          dgate[i * dir * c.ld_dgate] =
              Elem<T>::put(settled(decay<FORM>(a[i][0]).slope(sum[i])));
  }

  // offsets have to ascend from 0 to the tokens: each is looked at once
  if (c.offsets)
    for (int64_t i = (int64_t)blockIdx.x * kBlock + t; i <= c.nseq; i += (int64_t)gridDim.x * kBlock) {
      const int o = seq_offset(c, (int)i);
      const int next = i < c.nseq ? seq_offset(c, (int)i + 1) : c.tokens;
      if ((i == 0 && o != 0) || next < o || (i == c.nseq && o != c.tokens))
        atomicOr(c.flag, kFlagBadOffset);
    }
  // Whoever took the tile's last chunk makes the counters ready for the next launch: all
  // of them move on with every launch, so that a tag is one launch's.
  if (t == 0 && p.head && chunk == p.chunks - 1) {
    const uint32_t next = max(tag + 1, 1u);
    const int last = tile == 0 ? p.counters : tile + 1;
    for (int i = tile; i < last; i = i == 0 ? p.tiles : i + 1)
      __hip_atomic_store(p.head + i * kHeadLine, (uint64_t)next << 32, __ATOMIC_RELAXED,
                         __HIP_MEMORY_SCOPE_AGENT);
  }
}

// One token for every sequence: nothing to scan.  A thread per four channels; 64
// sequences of 256 bfloat16 channels take 2.9 us, or 2.0 each in a graph of many: a launch
// and one round trip.
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
      float da, rest;
      gate_pair<FORM>(gv, da, rest);
      o[v] = __fmaf_rn(da, h.get(v), rest * x.get(v));
    }
    store_quad<T, VEC>(static_cast<T*>(c.out) + n * c.ld_out + ch, o, nv);
    if (c.fin) store_quad<float, VEC>(c.fin + at, o, nv);
  }
}

}  // namespace pg
