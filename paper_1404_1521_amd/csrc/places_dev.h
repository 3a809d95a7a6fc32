// Packed sequences: where they start and stop among the tokens of a tile.
#pragma once
#include "common.h"
#include "operators.h"

namespace pg {

// Offset i of nseq + 1, held to [0, tokens]: no offset, whatever it holds, leads out of
// the tensors.
__device__ __forceinline__ int place_of(const Packed& s, int i) {
  if (!s.offsets) return i * (s.tokens / s.nseq);
  if (s.offset_bytes == 4)
    return min(max(static_cast<const int32_t*>(s.offsets)[i], 0), s.tokens);
  const int64_t o = static_cast<const int64_t*>(s.offsets)[i];
  return (int)min(max(o, (int64_t)0), (int64_t)s.tokens);
}

// The first of the offsets that is >= lo (nseq + 1 if none is), found by a whole wave:
// 64 probes split the range into 65 parts.
__device__ __forceinline__ int first_place(const Packed& s, int lo) {
  if (!s.offsets) return first_equal(lo, s.tokens / s.nseq);
  int l = 0, n = s.nseq + 1;  // the answer is in [l, l + n]
  while (n > 0) {
    const int step = ceil_div(n, kWave + 1);
    const int i = l + (lane_id() + 1) * step - 1;
    const bool below = i < l + n && place_of(s, i) < lo;
    const int k = __popcll(__ballot(below));  // of ascending offsets the first k are below
    l += k * step;
    n -= k * step;
    if (k < kWave) n = min(step - 1, n);  // the next probe is not below
  }
  return l;
}

// Where sequences start and stop in the tokens [lo, hi): by place, the sequence that
// starts or stops there or -1 (also in the places from hi - lo to `room`).  By a whole wave, with `cursor` the first
// offset >= lo.  Returns the first offset >= hi.  Offsets that do not ascend leave
// wrong sequences in the places, never one that is not there.
__device__ __forceinline__ int mark_places(const Packed& s, int lo, int hi, int room, int cursor,
                                           int* start, int* stop) {
  const int l = lane_id();
  for (int i = l; i < room; i += kWave) start[i] = stop[i] = -1;
  wave_lds_sync();
  int next = cursor;
  bool more = true;
  for (int base = cursor; more && base <= s.nseq; base += kWave) {
    const int i = base + l;
    const bool there = i <= s.nseq;
    const int o = there ? place_of(s, i) : INT32_MAX;
    if (there && o >= lo && o <= hi) {
      if (i < s.nseq && o < hi && place_of(s, i + 1) > o) start[o - lo] = i;
      if (i > 0 && o > lo && place_of(s, i - 1) < o) stop[o - 1 - lo] = i - 1;
    }
    const uint64_t below = __ballot(there && o < hi);
    if (below) next = base + (int)__popcll(below);
    // all of these lie in the tile or at its end: so may the next ones
    more = __ballot(there && o <= hi) == ~0ull;
  }
  wave_lds_sync();
  return next;
}

// The sequences' offsets near the tiles that a wave goes through, one to a lane: where none
// of them lies in a tile, which is the usual case in long sequences, nothing is read.
struct UpCursor {   // tiles in ascending order: the offsets from `at`, the first >= lo, on
  int at, o;
  __device__ __forceinline__ void read(const Packed& s, int first) {
    at = first;
    o = at + lane_id() <= s.nseq ? place_of(s, at + lane_id()) : INT32_MAX;
  }
};
struct DownCursor {  // in descending order: the offsets below `at`, the first > hi
  int at, o;
  __device__ __forceinline__ void read(const Packed& s, int first) {
    at = first;
    o = at - 1 - lane_id() >= 0 ? place_of(s, at - 1 - lane_id()) : -1;
  }
};

// The places of a tile and, as bits, where in it sequences start and stop.  By a whole wave;
// up to 32 places.
struct TileMarks {
  int start[32], stop[32];
  uint32_t starts, stops;
};
__device__ __forceinline__ void mark_bits(TileMarks& m) {
  const int l = lane_id() & 31;
  const uint32_t a = (uint32_t)__ballot(m.start[l] >= 0), b = (uint32_t)__ballot(m.stop[l] >= 0);
  m.starts = a;
  m.stops = b;
}
__device__ __forceinline__ void mark_tile(const Packed& s, int lo, int hi, UpCursor& c, TileMarks& m) {
  if (__ballot(c.o <= hi) == 0) {
    m.starts = m.stops = 0;
    return;
  }
  c.read(s, mark_places(s, lo, hi, 32, c.at, m.start, m.stop));
  mark_bits(m);
}
__device__ __forceinline__ void mark_tile(const Packed& s, int lo, int hi, DownCursor& c, TileMarks& m) {
  if (__ballot(c.o >= lo) == 0) {
    m.starts = m.stops = 0;
    return;
  }
  mark_places(s, lo, hi, 32, first_place(s, lo), m.start, m.stop);
  mark_bits(m);
  c.read(s, first_place(s, lo + 1));
}

// A workgroup's share of the sequences, the `part`-th of `parts`: raises the flag where
// the offsets do not ascend from 0 to the tokens, and calls copy(i) with every thread for
// each empty sequence i.  list: a place for each thread and one more.
template <class F>
__device__ __forceinline__ void check_places(const Packed& s, int part, int parts, int threads,
                                             bool copies, int* list, F copy) {
  const int t = threadIdx.x;
  for (int64_t base = (int64_t)part * threads; base < s.nseq; base += (int64_t)parts * threads) {
    if (copies && t == 0) list[threads] = 0;
    if (copies) __syncthreads();
    const int i = (int)base + t;
    if (i < s.nseq) {
      const int o = place_of(s, i), e = place_of(s, i + 1);
      bool bad = e < o || (i == 0 && o != 0) || (i == s.nseq - 1 && e != s.tokens);
      if (s.offsets && s.offset_bytes == 8) {
        const int64_t* p = static_cast<const int64_t*>(s.offsets) + i;
        bad |= p[0] < 0 || p[1] < 0 || p[0] > s.tokens || p[1] > s.tokens;
      } else if (s.offsets) {
        const int32_t* p = static_cast<const int32_t*>(s.offsets) + i;
        bad |= p[0] < 0 || p[1] < 0 || p[0] > s.tokens || p[1] > s.tokens;
      }
      if (bad) atomicOr(s.flag, kFlagBadOffset);
      if (copies && o == e) list[atomicAdd(&list[threads], 1)] = i;
    }
    if (!copies) continue;
    __syncthreads();
    const int n = __builtin_amdgcn_readfirstlane(list[threads]);
    for (int j = 0; j < n; ++j) copy(__builtin_amdgcn_readfirstlane(list[j]));
    __syncthreads();
  }
}

}  // namespace pg
