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

// How a call is cut, in the workspace.
inline SelPlan selective_plan(int64_t tokens, int D, int N, int groups, const SelSpace& space) {
  SelPlan p{};
  const int CB = sel_channels(sel_lanes(N));
  p.blocks = ceil_div(D / groups, CB);
  p.all_blocks = p.blocks * groups;
  const int64_t tiles = std::max<int64_t>(1, (tokens + kSelectiveTile - 1) / kSelectiveTile);
  const int64_t want = std::min<int64_t>(tiles, std::max(1, kSelWorkgroups / p.all_blocks));
  const int64_t each = (tiles + want - 1) / want;
  p.range = (int)(each * kSelectiveTile);
  p.ranges = (int)((tiles + each - 1) / each);
  p.NM = (N + 3) / 4 * 4;
  p.states = space.states;
  p.sums = space.sums;
  p.info = space.info;
  p.part_a = space.part_a;
  p.part_s = space.part_s;
  p.part_bc = space.part_bc;
  return p;
}

}  // namespace pg
