// Launches of the gated linear recurrence.
#include "operators.h"

#include <algorithm>

#include "recurrence_dev.h"

namespace pg {

namespace {

// Lanes of a row of threads: as few as hold all channels, so that narrow layers
// have more rows of tokens; at least what a group takes.
ScanPlan scan_plan(int64_t tokens, int D, int group, int R) {
  ScanPlan p{};
  p.lanes_per_group = group > 1 ? ceil_div(group, 4) : 1;
  const int64_t lanes = group > 1 ? (int64_t)p.lanes_per_group * (D / group) : ceil_div(D, 4);
  int log2 = 3;
  while (log2 < 6 && (1 << log2) < lanes) ++log2;
  p.lanes_log2 = log2;
  const int CT = 1 << log2;
  p.groups_per_tile = CT / p.lanes_per_group;
  p.tiles = group > 1 ? ceil_div(D / group, p.groups_per_tile) : ceil_div(D, 4 * CT);
  const int L = (kBlock / CT) * R;
  p.chunks = std::max(1, (int)((tokens + L - 1) / L));
  return p;
}

template <class T, int FORM, bool GRAD>
hipError_t launch_scan(const RecCall& c, uint64_t* head, uint64_t* words, size_t stride,
                       const Launch& L) {
  constexpr int R = scan_tokens<T, GRAD>();
  static_assert(kScanMaxRows * R <= kScanMaxTokens, "places of a chunk");
  ScanPlan p = scan_plan(c.tokens, c.D, c.group, R);
  p.head = head;
  p.words = words;
  p.stride = stride;
  const bool shared = c.group > 1;
  const bool vec = shared ? c.group % 4 == 0 : c.D % 4 == 0;  // whole quads
  auto k = shared ? (vec ? k_scan<T, FORM, GRAD, true, true, R> : k_scan<T, FORM, GRAD, true, false, R>)
                  : (vec ? k_scan<T, FORM, GRAD, false, true, R>
                         : k_scan<T, FORM, GRAD, false, false, R>);
  return pg_launch(k, dim3(p.chunks * p.tiles), dim3(kBlock), 0, L, c, p);
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

// Lanes that a group leaves idle at most double the slots (a group of two channels in
// a lane of four; 33 lanes of 64).
int scan_tiles(int D) { return ceil_div(2 * D, 4 * kWave) + 1; }

size_t scan_stride(int64_t tokens) {
  const int64_t L = kBlock / kWave * 8;  // chunks are shortest where a row has 64 lanes
  return (size_t)((tokens + L - 1) / L + 1) * (2 * 4 * kWave);
}

hipError_t launch_recurrence(const RecCall& c, int dtype, int form, bool grad, uint64_t* head,
                             uint64_t* words, size_t stride, const Launch& L) {
  constexpr int raw = POLYGLOT_GATE_RAW, sig = POLYGLOT_GATE_SIGMOID;
  const bool single = !c.offsets && c.tokens == c.nseq;  // every token starts a sequence
  return by_format(dtype, [&](auto v) {
    using T = decltype(v);
    if (single && !grad)
      return form == raw ? launch_step<T, raw>(c, L) : launch_step<T, sig>(c, L);
    uint64_t* h = single ? nullptr : head;
    if (grad)
      return form == raw ? launch_scan<T, raw, true>(c, h, words, stride, L)
                         : launch_scan<T, sig, true>(c, h, words, stride, L);
    return form == raw ? launch_scan<T, raw, false>(c, h, words, stride, L)
                       : launch_scan<T, sig, false>(c, h, words, stride, L);
  });
}

}  // namespace pg
