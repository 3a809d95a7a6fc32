// The best continuations of groups of beams, and the reordering of states that they ask for.
//
// A key is a candidate's sum, as an unsigned number that ascends with it, over the
// complement of its place: larger keys are larger sums, and of equal ones the lower place.
// No two candidates have the same key, so that the picks do not depend on who finds them.
//
// A workgroup takes a part of a row into registers, E words to a thread.  The k-th largest of
// the 256 threads' largest keys is a bound: the k picks are not below it, and only k threads
// hold keys that are not, k E at most.  Those go to a list, a few more than k as a rule, whose
// k largest, found by counting how many are larger, go out.  A second launch does the same
// over a group's parts, a batch at a time.
//
// 32 groups of 8 rows of 32,003 bfloat16 words, 16 picks: 13 us and 6 for the join, where the
// 16 MB take 3 at a copy's rate; what it waits for are the loads, then the bound, the list and
// its order one after the other.  A bound for each wave alone left longer lists (28 us for 19
// in all), and lists that waves keep in order took 27.
#pragma once
#include "logits_dev.h"
#include "operators.h"

namespace pg {

// -0 counts as +0; what is not to be picked (NaN, -infinity) has no key.
__device__ __forceinline__ uint64_t beam_key(float v, uint32_t place) {
  const uint32_t u = __float_as_uint(v + 0.f);
  if (!(v > -__builtin_inff())) return 0;
  return (uint64_t)(u & 0x80000000u ? ~u : u | 0x80000000u) << 32 | ~place;
}
__device__ __forceinline__ float beam_value(uint64_t key) {
  const uint32_t u = (uint32_t)(key >> 32);
  return __uint_as_float(u & 0x80000000u ? u & 0x7fffffffu : ~u);
}

__device__ __forceinline__ uint64_t lane_key(uint64_t v, int lane) {
  const uint32_t lo = __builtin_amdgcn_readlane((int)(uint32_t)v, lane);
  const uint32_t hi = __builtin_amdgcn_readlane((int)(uint32_t)(v >> 32), lane);
  return (uint64_t)hi << 32 | lo;
}
template <int LIST>
struct BeamLds {
  uint64_t best[kWavesPerBlock][kBeamPicks];  // of each wave the k largest of its lanes' largest
  uint64_t list[LIST];
  uint64_t bound;
  int n;
};

// The k-th largest of the threads' keys `best` (0 where there are fewer).  First in each wave
// by its lanes one after the other, then among the waves' k largest.  Ends on a barrier; the
// list is empty then.
template <int LIST>
__device__ __forceinline__ uint64_t group_bound(uint64_t best, int k, BeamLds<LIST>& l) {
  const int lane = lane_id(), wave = threadIdx.x / kWave;
  int above = 0;
#pragma unroll 16
  for (int i = 0; i < kWave; ++i) above += lane_key(best, i) > best;
  if (lane < k) l.best[wave][lane] = 0;
  if (threadIdx.x == 0) l.n = 0, l.bound = 0;
  wave_lds_sync();
  if (best && above < k) l.best[wave][above] = best;
  __syncthreads();
  if (best && above < k) {
    int rank = above;
#pragma unroll
    for (int w = 1; w < kWavesPerBlock; ++w) {
      const uint64_t* other = l.best[(wave + w) % kWavesPerBlock];
#pragma unroll 4
      for (int i = 0; i < k; ++i) rank += other[i] > best;
    }
    if (rank == k - 1) l.bound = best;  // one thread: keys differ
  }
  __syncthreads();
  return l.bound;
}

// The k largest of the list, to out[k] in their order (0: none).
template <int LIST>
__device__ __forceinline__ void rank_list(const BeamLds<LIST>& l, int k, uint64_t* out) {
  const int n = l.n;
  for (int i = threadIdx.x; i < n; i += kBlock) {
    const uint64_t own = l.list[i];
    int rank = 0, j = 0;
    for (; j + 8 <= n && rank < k; j += 8) {
#pragma unroll
      for (int e = 0; e < 8; ++e) rank += l.list[j + e] > own;
    }
    for (; j < n; ++j) rank += l.list[j] > own;
    if (rank < k) out[rank] = own;
  }
  for (int i = n + threadIdx.x; i < k; i += kBlock) out[i] = 0;
}

// E words to a thread, in quads 4 * 256 words apart.
template <class T, int E>
__global__ __launch_bounds__(kBlock) void k_beam_parts(BeamCall c) {
  __shared__ BeamLds<kBeamPicks * E> l;
  const int t = threadIdx.x;
  const int64_t r = blockIdx.x / c.parts;
  const int part = (int)(blockIdx.x - r * c.parts);
  uint64_t* out = c.keys + (int64_t)blockIdx.x * c.picks;
  const float total = c.total[r];
  if (c.finished && c.finished[r]) {  // its one candidate: nothing more is said
    const bool here = c.end / (E * kBlock) == part;
    for (int i = t; i < c.picks; i += kBlock)
      out[i] = i == 0 && here ? beam_key(total, (uint32_t)c.end) : 0;
    return;
  }
  const int v0 = part * (E * kBlock) + 4 * t;
  const bool whole = (part + 1) * (E * kBlock) <= c.V;
  const T* in = static_cast<const T*>(c.scores) + r * c.ld;
  Quad<T> x[E / 4];
#pragma unroll
  for (int g = 0; g < E / 4; ++g) x[g] = row_quad<T>(in, v0 + g * 4 * kBlock, c.V, whole);
  const float base = c.lse ? __fsub_rn(total, c.lse[r]) : total;
  const auto place = [&](int i) { return (i / 4) * 4 * kBlock + (i & 3); };
  const auto sum = [&](int i) {
    const float v = __fadd_rn(x[i / 4].get(i & 3), base);
    return whole || v0 + place(i) < c.V ? v : -__builtin_inff();
  };
  // the largest sum, and the first place that has it
  float top = -__builtin_inff();
#pragma unroll
  for (int i = 0; i < E; ++i) top = fmaxf(top, sum(i));  // (not a NaN)
  int first = 0;
#pragma unroll
  for (int i = E - 1; i >= 0; --i)
    if (sum(i) == top) first = place(i);
  const uint64_t best = beam_key(top, (uint32_t)(v0 + first));
  const uint64_t bound = group_bound(best, c.picks, l);
  if (best >= bound && best) {
    const float low = bound ? beam_value(bound) : -__builtin_inff();
#pragma unroll
    for (int i = 0; i < E; ++i) {
      const float v = sum(i);
      if (!(v >= low)) continue;
      const uint64_t key = beam_key(v, (uint32_t)(v0 + place(i)));
      if (key && key >= bound) l.list[atomicAdd(&l.n, 1)] = key;
    }
  }
  __syncthreads();
  rank_list(l, c.picks, out);
}

// A workgroup for each group: its rows' parts, 256 E keys at a time beside the picks so far.
template <int E>
__global__ __launch_bounds__(kBlock) void k_beam_join(BeamCall c) {
  __shared__ BeamLds<kBeamPicks * (E + 1)> l;
  __shared__ uint64_t picks[kBeamPicks];
  const int t = threadIdx.x;
  const int64_t row0 = (int64_t)blockIdx.x * c.beams;
  const int64_t each = (int64_t)c.parts * c.picks, all = each * c.beams;
  const uint64_t* in = c.keys + row0 * each;
  if (t < kBeamPicks) picks[t] = 0;
  __syncthreads();
  for (int64_t first = 0; first < all; first += E * kBlock) {
    uint64_t key[E + 1], best = 0;
#pragma unroll
    for (int i = 0; i < E; ++i) {
      const int64_t at = first + i * kBlock + t;
      key[i] = at < all ? in[at] : 0;
    }
#pragma unroll
    for (int i = 0; i < E; ++i) {
      const int64_t at = first + i * kBlock + t;
      if (key[i]) {  // the place in a row becomes the place in the group
        const uint32_t b = all < (1ll << 32) ? (uint32_t)at / (uint32_t)each : (uint32_t)(at / each);
        key[i] = (key[i] & 0xffffffff00000000ull) | ~(~(uint32_t)key[i] + b * (uint32_t)c.V);
      }
      best = key[i] > best ? key[i] : best;
    }
    if (!__syncthreads_or(best > picks[c.picks - 1])) continue;
    key[E] = t < c.picks ? picks[t] : 0;
    best = key[E] > best ? key[E] : best;
    const uint64_t bound = group_bound(best, c.picks, l);
    if (best >= bound && best) {
#pragma unroll
      for (int i = 0; i <= E; ++i)
        if (key[i] && key[i] >= bound) l.list[atomicAdd(&l.n, 1)] = key[i];
    }
    __syncthreads();
    rank_list(l, c.picks, picks);
    __syncthreads();
  }
  if (t >= c.picks) return;
  const int64_t o = (int64_t)blockIdx.x * c.picks + t;
  const uint64_t key = picks[t];
  const uint32_t place = ~(uint32_t)key;
  const uint32_t b = key ? place / (uint32_t)c.V : (uint32_t)(t % c.beams);
  c.parent[o] = (int32_t)(row0 + b);
  c.token[o] = key ? (int32_t)(place - b * (uint32_t)c.V) : -1;
  c.out[o] = key ? beam_value(key) : -__builtin_inff();
}

// out[r] = in[ids[r]] for several tensors in one launch: a workgroup copies a piece of 16 KB of a
// row, four loads of 16 bytes to a thread on their way at once.  Memory bounds it: 256 rows of
// 17 tensors, 587 MB read and written, in 86 us, 6.8 TB/s; two narrow layers take 3.8, a launch.
__global__ __launch_bounds__(kBlock) void k_reorder(ReorderCall c) {
  int64_t piece = blockIdx.x;
  const int64_t all = c.first[c.count];
  for (; piece < all; piece += gridDim.x) {
    int k = 0;
    while (k + 1 < c.count && piece >= c.first[k + 1]) ++k;
    const RowCopy& m = c.item[k];
    const int64_t local = piece - c.first[k];
    const int64_t r = local / m.pieces;
    const int64_t from = (local - r * m.pieces) * kReorderPiece;
    const int64_t bytes = min((int64_t)kReorderPiece, m.row_bytes - from);
    const int32_t id = c.ids[r];
    if ((uint32_t)id >= (uint32_t)m.in_rows) {
      if (threadIdx.x == 0) atomicOr(c.flag, kFlagBadId);
      continue;
    }
    const char* in = m.in + id * m.ld_in + from;
    char* out = m.out + r * m.ld_out + from;
    const int t = threadIdx.x;
    if (m.unit == 16) {
      const int n = (int)(bytes / 16);
      uint4 v[kReorderPiece / (16 * kBlock)];
#pragma unroll
      for (int i = 0; i < kReorderPiece / (16 * kBlock); ++i)
        v[i] = t + i * kBlock < n ? reinterpret_cast<const uint4*>(in)[t + i * kBlock] : uint4{};
#pragma unroll
      for (int i = 0; i < kReorderPiece / (16 * kBlock); ++i)
        if (t + i * kBlock < n) reinterpret_cast<uint4*>(out)[t + i * kBlock] = v[i];
    } else if (m.unit == 4) {
      const int n = (int)(bytes / 4);
#pragma unroll 4
      for (int i = t; i < n; i += kBlock)
        reinterpret_cast<uint32_t*>(out)[i] = reinterpret_cast<const uint32_t*>(in)[i];
    } else if (m.unit == 2) {
      const int n = (int)(bytes / 2);
#pragma unroll 4
      for (int i = t; i < n; i += kBlock)
        reinterpret_cast<uint16_t*>(out)[i] = reinterpret_cast<const uint16_t*>(in)[i];
    } else {
#pragma unroll 4
      for (int i = t; i < (int)bytes; i += kBlock) out[i] = in[i];
    }
  }
}

}  // namespace pg
