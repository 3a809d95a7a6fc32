// Launches of the selective scan and its gradient.
#include "operators.h"

#include <algorithm>
#include <type_traits>

#include "selective_grad_dev.h"

namespace pg {

namespace {

// Lanes of a channel: four states each.
int sel_lanes(int N) { return N <= 8 ? 2 : N <= 16 ? 4 : N <= 32 ? 8 : 16; }

template <class T, int LN>
hipError_t forward(const SelCall& c, SelPlan p, const Launch& L) {
  const dim3 grid((uint32_t)p.ranges * p.all_blocks);
  if (p.ranges > 1) {
    const hipError_t e = pg_launch(k_selective_ends<T, LN>, grid, dim3(kBlock), 0, L, c, p);
    if (e != hipSuccess) return e;
  }
  return pg_launch(k_selective<T, LN>, grid, dim3(kBlock), 0, L, c, p);
}

template <class T, int LN>
hipError_t backward(const SelCall& c, SelPlan p, const Launch& L) {
  const dim3 grid((uint32_t)p.ranges * p.all_blocks);
  hipError_t e = hipSuccess;
  if (p.ranges > 1) e = pg_launch(k_selective_grad_ends<T, LN>, grid, dim3(kBlock), 0, L, c, p);
  if (e == hipSuccess) e = pg_launch(k_selective_grad<T, LN>, grid, dim3(kBlock), 0, L, c, p);
  if (e != hipSuccess) return e;
  const int params = (int)(((int64_t)c.D * (c.N + 2) + kWave - 1) / kWave);
  const int64_t rest = p.blocks == 1 ? 0 : (int64_t)c.groups * 2 * c.N * c.seqs.tokens;
  const int sums = (int)std::min<int64_t>((rest + kBlock - 1) / kBlock, 16 * kCus);
  return pg_launch(k_selective_sums<T>, dim3(params + sums), dim3(kBlock), 0, L, c, p, 4 * LN, params);
}

template <class T, int LN>
hipError_t step(const SelCall& c, const Launch& L) {
  const int blocks = ceil_div(c.D, kBlock / LN);
  const int64_t grid = std::min<int64_t>((int64_t)c.seqs.nseq * blocks, 1 << 20);
  return pg_launch(k_selective_step<T, LN>, dim3((uint32_t)grid), dim3(kBlock), 0, L, c, blocks);
}

template <class F>
hipError_t by_lanes(int N, F f) {
  switch (sel_lanes(N)) {
    case 2: return f(std::integral_constant<int, 2>{});
    case 4: return f(std::integral_constant<int, 4>{});
    case 8: return f(std::integral_constant<int, 8>{});
    default: return f(std::integral_constant<int, 16>{});
  }
}

constexpr int kSelWorkgroups = 2 * kCus;  // that the ranges are to give

// How a call is cut; the workspace's pointers are left to selective_room.
SelPlan selective_plan(int64_t tokens, int D, int N, int groups) {
  SelPlan p{};
  const int CB = 512 / sel_lanes(N);
  p.blocks = ceil_div(D / groups, CB);
  p.all_blocks = p.blocks * groups;
  const int64_t tiles = std::max<int64_t>(1, (tokens + kSelectiveTile - 1) / kSelectiveTile);
  const int64_t want = std::min<int64_t>(tiles, std::max(1, kSelWorkgroups / p.all_blocks));
  const int64_t each = (tiles + want - 1) / want;
  p.range = (int)(each * kSelectiveTile);
  p.ranges = (int)((tiles + each - 1) / each);
  p.NM = (N + 3) / 4 * 4;
  return p;
}

// Channels times ranges of any call of up to D channels: one range, or as many as give
// the workgroups of up to CB channels.
int64_t range_channels(int D, int N) {
  return std::max<int64_t>(D, (int64_t)kSelWorkgroups * (512 / sel_lanes(N)));
}

}  // namespace

SelRoom selective_room(int64_t tokens, int D, int N) {
  // Fewer states have fewer lanes and wider workgroups: the sizes below grow with N, but for
  // the channels of a workgroup, which are taken at their most.
  SelRoom r;
  const int LN = sel_lanes(N), NP = 4 * LN;
  const int64_t rc = range_channels(D, 1);
  r.states = (size_t)rc * NP;
  r.sums = (size_t)rc;
  r.info = (size_t)std::max<int64_t>(kSelWorkgroups, 1);
  r.part_s = 2 * (size_t)rc;
  // blocks of a head's channels, where there are two or more: at most twice D / CB
  r.part_bc = (size_t)tokens * 2 * N * (2 * (size_t)D / (512 / LN) + 2);
  return r;
}

hipError_t launch_selective(const SelCall& c, int dtype, SelSpace space, const Launch& L) {
  const int64_t T = c.seqs.tokens;
  SelPlan p = selective_plan(T, c.D, c.N, c.groups);
  p.states = space.states;
  p.sums = space.sums;
  p.info = space.info;
  return by_format(dtype, [&](auto v) {
    using E = decltype(v);
    return by_lanes(c.N, [&](auto ln) { return forward<E, decltype(ln)::value>(c, p, L); });
  });
}

hipError_t launch_selective_grad(const SelCall& c, int dtype, SelSpace space, const Launch& L) {
  SelPlan p = selective_plan(c.seqs.tokens, c.D, c.N, c.groups);
  p.states = space.states;
  p.sums = space.sums;
  p.info = space.info;
  p.part_a = space.part_a;
  p.part_s = space.part_s;
  p.part_bc = space.part_bc;
  return by_format(dtype, [&](auto v) {
    using E = decltype(v);
    return by_lanes(c.N, [&](auto ln) { return backward<E, decltype(ln)::value>(c, p, L); });
  });
}

hipError_t launch_selective_step(const SelCall& c, int dtype, const Launch& L) {
  return by_format(dtype, [&](auto v) {
    using E = decltype(v);
    return by_lanes(c.N, [&](auto ln) { return step<E, decltype(ln)::value>(c, L); });
  });
}

}  // namespace pg
