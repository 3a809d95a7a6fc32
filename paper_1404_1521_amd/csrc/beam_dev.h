// The best continuations of groups of beams, and the reordering of states that they ask for.
//
// A key is a candidate's sum, as an unsigned number that ascends with it, over the
// complement of its place: larger keys are larger sums, and of equal ones the lower place.
// No two candidates have the same key, so that the picks do not depend on who finds them.
//
// A wave keeps the k largest keys that it has met, the i-th largest in lane i, and looks a
// batch of its words over: sums, the lanes' largest, and only where one of those is above the
// wave's k-th is a word taken in, by its rank among the lanes.  Of its first batch the k-th
// largest of the 64 lanes' largest keys is a bound already.  The four waves' keys are ranked by
// counting how many are larger; a second launch does the same with the parts of a group.
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
// The k-th largest of a wave's keys `best` (0 where there are fewer).
__device__ __forceinline__ uint64_t wave_bound(uint64_t best, int k) {
  int above = 0;
#pragma unroll 16
  for (int i = 0; i < kWave; ++i) above += lane_key(best, i) > best;
  const uint64_t at = __ballot(above == k - 1 && best);  // one lane: keys differ
  return at ? lane_key(best, __builtin_ctzll(at)) : 0;
}
__device__ __forceinline__ uint32_t lane_before(uint32_t v) {  // the lane before's (DPP wave_shr:1)
  return (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, 0x138, 0xf, 0xf, false);
}

// A wave's k largest keys.
struct WaveBest {
  uint64_t held = 0;   // of lane i the i-th largest
  uint64_t least = 1;  // a key has to be no smaller to be taken in
  int k;
  __device__ __forceinline__ explicit WaveBest(int k) : k(k) {}
  // What the lanes bring: none of them has a key above `best`.
  __device__ __forceinline__ void begin(uint64_t best) {
    const uint64_t b = wave_bound(best, k);
    if (b > least) least = b;
  }
  // Takes the lanes' keys in where `want`.
  __device__ __forceinline__ void take(uint64_t key, bool want) {
    uint64_t lanes = __ballot(want && key >= least);
    while (lanes) {
      const int l = __builtin_ctzll(lanes);
      lanes &= lanes - 1;
      const uint64_t own = lane_key(key, l);
      const int rank = __popcll(__ballot(held > own));
      if (rank >= k) continue;
      const uint64_t before = (uint64_t)lane_before((uint32_t)(held >> 32)) << 32 | lane_before((uint32_t)held);
      const int lane = lane_id();
      held = lane < rank ? held : lane == rank ? own : before;
      const uint64_t last = lane_key(held, k - 1);
      if (last > least) least = last;
    }
  }
};

// The workgroup's k largest of its waves' to out[k], in their order (0: none).
__device__ __forceinline__ void join_waves(const WaveBest& w, int k, uint64_t* list, uint64_t* out) {
  const int lane = lane_id(), wave = threadIdx.x / kWave;
  if (lane < k) list[wave * k + lane] = w.held;
  __syncthreads();
  const int n = kWavesPerBlock * k;
  if ((int)threadIdx.x >= n) return;
  const uint64_t own = list[threadIdx.x];
  int rank = 0;
  for (int j = 0; j < n; j += 4) {
#pragma unroll
    for (int e = 0; e < 4; ++e) rank += list[j + e] > own || (list[j + e] == own && j + e < (int)threadIdx.x);
  }
  if (rank < k) out[rank] = own;  // (no keys, 0, are ranked by their places)
}

constexpr int kBeamBatch = 16;  // words of a thread at a time, in quads 4 * 256 words apart

template <class T>
__global__ __launch_bounds__(kBlock) void k_beam_parts(BeamCall c) {
  constexpr int E = kBeamBatch;
  __shared__ uint64_t list[kWavesPerBlock * kBeamPicks];
  const int t = threadIdx.x;
  const int64_t r = blockIdx.x / c.parts;
  const int part = (int)(blockIdx.x - r * c.parts);
  uint64_t* out = c.keys + (int64_t)blockIdx.x * c.picks;
  const int begin = (int)min((int64_t)part * c.part_words, (int64_t)c.V);
  const int end = (int)min((int64_t)begin + c.part_words, (int64_t)c.V);
  const float total = c.total[r];
  if (c.finished && c.finished[r]) {  // its one candidate: nothing more is said
    const bool here = c.end >= begin && c.end < end;
    for (int i = t; i < c.picks; i += kBlock)
      out[i] = i == 0 && here ? beam_key(total, (uint32_t)c.end) : 0;
    return;
  }
  const T* in = static_cast<const T*>(c.scores) + r * c.ld;
  Quad<T> next[E / 4];
  const auto fetch = [&](int v0) {
    const bool whole = v0 + E * kBlock <= c.V;
#pragma unroll
    for (int g = 0; g < E / 4; ++g) next[g] = row_quad<T>(in, v0 + 4 * t + g * 4 * kBlock, c.V, whole);
  };
  if (begin < end) fetch(begin);
  const float base = c.lse ? __fsub_rn(total, c.lse[r]) : total;
  WaveBest best(c.picks);
  for (int v0 = begin; v0 < end; v0 += E * kBlock) {
    float v[E], top = -__builtin_inff();
    const bool whole = v0 + E * kBlock <= end;
#pragma unroll
    for (int i = 0; i < E; ++i) {
      v[i] = __fadd_rn(next[i / 4].get(i & 3), base);
      if (!whole && v0 + 4 * t + (i / 4) * 4 * kBlock + (i & 3) >= end) v[i] = -__builtin_inff();
      top = fmaxf(top, v[i]);  // (not a NaN)
    }
    if (v0 + E * kBlock < end) fetch(v0 + E * kBlock);
    const auto place = [&](int i) { return (uint32_t)(v0 + 4 * t + (i / 4) * 4 * kBlock + (i & 3)); };
    if (v0 == begin) {
      int first = 0;
#pragma unroll
      for (int i = E - 1; i >= 0; --i)
        if (v[i] == top) first = i;
      best.begin(beam_key(top, (uint32_t)(v0 + 4 * t + (first / 4) * 4 * kBlock + (first & 3))));
    }
    const float low = best.least > 1 ? beam_value(best.least) : -__builtin_inff();
    if (!__ballot(top >= low)) continue;
#pragma unroll
    for (int i = 0; i < E; ++i)
      if (__ballot(v[i] >= low)) best.take(beam_key(v[i], place(i)), v[i] >= low);
  }
  join_waves(best, c.picks, list, out);
}

// A workgroup for each group: its rows' parts.
__global__ __launch_bounds__(kBlock) void k_beam_join(BeamCall c) {
  constexpr int E = 8;
  __shared__ uint64_t list[kWavesPerBlock * kBeamPicks], picks[kBeamPicks];
  const int t = threadIdx.x;
  const int64_t row0 = (int64_t)blockIdx.x * c.beams;
  const int64_t each = (int64_t)c.parts * c.picks, all = each * c.beams;
  const uint64_t* in = c.keys + row0 * each;
  WaveBest best(c.picks);
  for (int64_t first = 0; first < all; first += E * kBlock) {
    uint64_t key[E], top = 0;
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
      top = key[i] > top ? key[i] : top;
    }
    if (first == 0) best.begin(top);
#pragma unroll
    for (int i = 0; i < E; ++i) best.take(key[i], true);
  }
  join_waves(best, c.picks, list, picks);
  __syncthreads();
  if (t >= c.picks) return;
  const int64_t o = (int64_t)blockIdx.x * c.picks + t;
  const uint64_t key = picks[t];
  const uint32_t place = ~(uint32_t)key;
  const uint32_t b = key ? place / (uint32_t)c.V : (uint32_t)(t % c.beams);
  c.parent[o] = (int32_t)(row0 + b);
  c.token[o] = key ? (int32_t)(place - b * (uint32_t)c.V) : -1;
  c.out[o] = key ? beam_value(key) : -__builtin_inff();
}

// out[r] = in[ids[r]] for several tensors: a workgroup copies pieces of rows.
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
