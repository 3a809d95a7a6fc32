// How selective scans are cut into workgroups; the kernel's lanes by the states.
#pragma once
#include <algorithm>
#include <type_traits>

#include "operators.h"

namespace pg {

template <class F>
hipError_t by_lanes(int N, F f) {
  switch (sel_lanes(N)) {
    case 2: return f(std::integral_constant<int, 2>{});
    case 4: return f(std::integral_constant<int, 4>{});
    case 8: return f(std::integral_constant<int, 8>{});
    default: return f(std::integral_constant<int, 16>{});
  }
}

constexpr int kSelWorkgroups = 4 * kCus;  // that the ranges are to give
constexpr int kSelFewRanges = 2 * kSelGroup;  // of a sequence

// How a call is cut, in the workspace.
inline SelPlan selective_plan(int64_t tokens, int nseq, int D, int N, int groups, const SelSpace& space) {
  SelPlan p{};
  const int CB = sel_channels(sel_lanes(N));
  p.blocks = ceil_div(D / groups, CB);
  p.all_blocks = p.blocks * groups;
  const int64_t tiles = std::max<int64_t>(1, (tokens + kSelectiveTile - 1) / kSelectiveTile);
  p.ranges = (int)std::min<int64_t>(tiles, std::max(1, kSelWorkgroups / p.all_blocks));
  p.share = Shares(tiles, p.ranges);
  p.NM = (N + 3) / 4 * 4;
  // A range takes those before it in its sequence in one after the other, 0.2 us each; where
  // they are many, groups of them are put together first, a launch of 5 us: one sequence of
  // 16,384 x 64 forward 295 -> 75 us and four of 4,096 x 256 (64 ranges each) 49 -> 39, but one
  // of 16,384 x 2,048 (64 ranges) 289 -> 294 and 700 of 16,384 x 256 46 -> 56.
  p.groups = p.ranges > kSelFewRanges * (int64_t)nseq ? (p.ranges + kSelGroup - 1) / kSelGroup : 0;
  const int64_t rows = (int64_t)p.ranges * D, NP = 4 * sel_lanes(N);
  p.group_states = space.states + rows * NP;
  p.group_sums = space.sums + rows;
  p.group_info = space.info + p.ranges;
  p.states = space.states;
  p.sums = space.sums;
  p.info = space.info;
  p.part_a = space.part_a;
  p.part_s = space.part_s;
  p.part_bc = space.part_bc;
  return p;
}

}  // namespace pg
