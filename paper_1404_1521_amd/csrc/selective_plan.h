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

// Workgroups that the ranges are to give: as many as run at once (half as many: 32,768 x 2,048
// bfloat16 683 us for 553 and back 1,472 for 1,380, 16,384 x 256 of 8 states 70 for 46), and
// up to twice as many where a range keeps kSelLongRange tiles: the chip is busy more evenly,
// 32,768 x 2,048 553 -> 535 and back 1,380 -> 1,350, 16,384 x 1,024 of 64 states 470 -> 441,
// but with four tiles to a range 16,384 x 1,024 of 4 states 123 -> 131 and 4,097 x 2,048
// 98 -> 103.  Four times as many: 547 and 1,371.
constexpr int kSelWorkgroups = 4 * kCus, kSelMostWorkgroups = 2 * kSelWorkgroups;
constexpr int kSelLongRange = 8;
constexpr int kSelFewRanges = 4 * kSelGroup;  // of a sequence

// How a call is cut, in the workspace.
inline SelPlan selective_plan(const Packed& seqs, int D, int N, int groups, const SelSpace& space) {
  SelPlan p{};
  const int64_t tokens = seqs.tokens;
  const int CB = sel_channels(sel_lanes(N));
  p.blocks = ceil_div(D / groups, CB);
  p.all_blocks = p.blocks * groups;
  const int64_t tiles = std::max<int64_t>(1, (tokens + kSelectiveTile - 1) / kSelectiveTile);
  const int few = std::max(1, kSelWorkgroups / p.all_blocks), most = std::max(1, kSelMostWorkgroups / p.all_blocks);
  p.ranges = (int)std::clamp<int64_t>(tiles / kSelLongRange, std::min<int64_t>(tiles, few), most);
  p.share = Shares(tiles, p.ranges);
  p.NM = (N + 3) / 4 * 4;
  // A range takes those before it in its sequence in one after the other, 0.2 us each; where
  // they may be many, groups of them are put together first, in a launch of 8 to 10 us, of 2
  // where no run of ranges is long enough to need it.  Offsets lie on the device: any of several
  // sequences may have nearly all ranges.  One long sequence beside 32 short ones, 16,384 x 64
  // (1,024 ranges), 270 -> 60 us forward and 305 -> 89 back, 16,384 x 256 165 -> 65 and 216 ->
  // 120; but 700 in 16,384 x 256 42 -> 44 and 80 -> 82.  At up to 128 ranges groups would cost
  // several even sequences what they save uneven ones: 2,048 x 64 25 -> 32, 44 -> 30; 32,768 x
  // 2,048 498 -> 505, 555 -> 527.  One sequence of 16,384 x 64 is 295 us without them, one of
  // 16,384 x 2,048 (64 ranges) 289, and 294 with them.
  const int64_t longest = seqs.nseq == 1 ? p.ranges : seqs.offsets ? p.ranges / 2 : p.ranges / seqs.nseq + 2;
  p.groups = longest > kSelFewRanges ? (p.ranges + kSelGroup - 1) / kSelGroup : 0;
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
