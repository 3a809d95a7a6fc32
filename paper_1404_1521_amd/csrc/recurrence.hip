// Launches of the gated linear recurrence.
#include "operators.h"

#include <algorithm>

#include "recurrence_dev.h"

namespace pg {

namespace {

// Lanes of a row of threads where a group of channels does not ask for more.  16 lanes
// of four channels are whole cache lines of 16-bit elements.  With 8 a narrow layer has
// twice the tiles, whose workgroups count themselves in side by side (10 ns each on one
// counter), and half the chunks to join; 8 lanes are whole lines of float32.  One sequence,
// sigmoid gates, us for 8 and 16 lanes, forward, gradient: 65,537 x 64 float32 25.7, 34.7
// and 28.6, 39.9; bfloat16 23.4, 33.1 and 23.8, 32.9; 16,384 x 512 float32 32.4, 50.4 and
// 35.5, 53.7; bfloat16 27.0, 44.8 and 24.9, 39.4; 65,536 x 2,048 float32 369, 718 and 376,
// 660; bfloat16 281, 541 and 246, 428 (32 lanes 262, 441).
int scan_lanes_log2(int D, size_t size) { return D <= 64 || (size == 4 && D <= 512) ? 3 : 4; }

// As few lanes as hold all channels, so that narrow layers have more rows of tokens; at
// least what a group takes.
ScanPlan scan_plan(int64_t tokens, int D, int group, int R, size_t size) {
  ScanPlan p{};
  p.lanes_per_group = group > 1 ? ceil_div(group, 4) : 1;
  const int64_t lanes = group > 1 ? (int64_t)p.lanes_per_group * (D / group) : ceil_div(D, 4);
  int log2 = 3;
  while (log2 < 6 && (1 << log2) < lanes &&
         (log2 < scan_lanes_log2(D, size) || (1 << log2) < p.lanes_per_group))
    ++log2;
  p.lanes_log2 = log2;
  const int CT = 1 << log2;
  p.groups_per_tile = CT / p.lanes_per_group;
  p.tiles = group > 1 ? ceil_div(D / group, p.groups_per_tile) : ceil_div(D, 4 * CT);
  const int L = kBlock / CT * R;
  p.chunks = std::max(1, (int)((tokens + L - 1) / L));
  p.group_log2 = log2 < 6 ? 4 : 3;  // kScanMateSlots
  return p;
}

template <class T, int FORM, bool GRAD, int R>
hipError_t launch_cut(const RecCall& c, ScanPlan p, const ScanSpace* space, const Launch& L) {
  if (space && p.chunks > 1) {  // one chunk waits for nobody
    p.counters = space->counters;
    p.head = space->head;
    p.flags = space->head + (size_t)space->counters * kHeadLine;
    p.words = p.flags + space->flags;
    const size_t groups = (p.chunks >> p.group_log2) + 1;
    if (p.tiles > space->counters || p.tiles * (p.chunks + groups) > space->flags ||
        (p.tiles * (8 * (size_t)p.chunks + 12 * groups) << p.lanes_log2) > space->words)
      return hipErrorInvalidValue;  // not reached within what scan_space bounds
  }
  const bool shared = c.group > 1;
  // Whole quads.  Otherwise every quad, not a row's last alone, is loaded and stored element
  // by element: sigmoid gates, forward and gradient, 16,384 x 509 bfloat16 42 and 97 us for
  // 26 and 39 at 512, float32 48 and 89 for 32 and 50; 65,536 x 2,047 bfloat16 627 and 1,219
  // for 242 and 428 at 2,048, float32 526 and 1,033 for 376 and 660.
  const bool vec = shared ? c.group % 4 == 0 : c.D % 4 == 0;
  auto k = shared ? (vec ? k_scan<T, FORM, GRAD, true, true, R>
                         : k_scan<T, FORM, GRAD, true, false, R>)
                  : (vec ? k_scan<T, FORM, GRAD, false, true, R>
                         : k_scan<T, FORM, GRAD, false, false, R>);
  return pg_launch(k, dim3(p.chunks * p.tiles), dim3(kBlock), 0, L, c, p);
}

template <class T, int FORM, bool GRAD>
hipError_t launch_scan(const RecCall& c, const ScanSpace* space, const Launch& L) {
  constexpr int R = scan_tokens<T, FORM, GRAD>();
  static_assert(R >= kScanMinTokens, "scan_space");
  const ScanPlan p = scan_plan(c.tokens, c.D, c.group, R, sizeof(T));
  if ((int64_t)p.chunks * p.tiles >= kScanFewWorkgroups)
    return launch_cut<T, FORM, GRAD, R>(c, p, space, L);
  return launch_cut<T, FORM, GRAD, kScanShortTokens>(
      c, scan_plan(c.tokens, c.D, c.group, kScanShortTokens, sizeof(T)), space, L);
}

template <class T, int FORM>
hipError_t launch_step(const RecCall& c, const Launch& L) {
  const bool vec = c.D % 4 == 0;
  const int64_t total = (int64_t)c.tokens * ceil_div(c.D, 4);
  const int grid = (int)std::min<int64_t>((total + kBlock - 1) / kBlock, 16 * kCus);
  return pg_launch(vec ? k_recurrence_step<T, FORM, true> : k_recurrence_step<T, FORM, false>,
                   dim3(grid), dim3(kBlock), 0, L, c);
}

}  // namespace

ScanSpace scan_space(int64_t tokens, int D) {
  // Lanes that a group leaves idle at most double the channels' slots (a group of two
  // channels in a lane of four; 33 lanes of 64), beside one tile's.  Rows of 64 lanes
  // have the shortest chunks, rows of 8 the narrowest tiles.
  const int64_t L = kBlock / kWave * kScanMinTokens, chunks = (tokens + L - 1) / L + 1;
  ScanSpace sp;
  sp.counters = ceil_div(2 * D, 4 * kScanMinLanes) + 1;
  const int64_t groups = chunks / 8 + 1;
  sp.flags = (size_t)(chunks + groups) * sp.counters;
  sp.words = (size_t)(2 * chunks + 3 * groups) * (2 * (size_t)D + 4 * kWave);
  // the short cut has up to four times the chunks of the few workgroups, and a tile's
  // last one and its group beside them
  const size_t few = 4 * kScanFewWorkgroups + 2 * (size_t)sp.counters;
  sp.flags += 2 * few;
  sp.words += 20 * few * kWave;
  return sp;
}

hipError_t launch_recurrence(const RecCall& c, int dtype, int form, bool grad,
                             const ScanSpace& space, const Launch& L) {
  constexpr int raw = POLYGLOT_GATE_RAW, sig = POLYGLOT_GATE_SIGMOID;
  const bool single = !c.offsets && c.tokens == c.nseq;  // every token starts a sequence
  return by_format(dtype, [&](auto v) {
    using T = decltype(v);
    if (single && !grad)
      return form == raw ? launch_step<T, raw>(c, L) : launch_step<T, sig>(c, L);
    const ScanSpace* sp = single ? nullptr : &space;
    if (grad)
      return form == raw ? launch_scan<T, raw, true>(c, sp, L)
                         : launch_scan<T, sig, true>(c, sp, L);
    return form == raw ? launch_scan<T, raw, false>(c, sp, L)
                       : launch_scan<T, sig, false>(c, sp, L);
  });
}

}  // namespace pg
