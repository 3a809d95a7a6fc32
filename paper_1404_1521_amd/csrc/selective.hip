// Launches of the selective scan.
#include "selective_dev.h"
#include "selective_plan.h"

namespace pg {

namespace {

template <class T, int LN>
hipError_t forward(const SelCall& c, const SelPlan& p, const Launch& L) {
  const dim3 block(SelShape<LN>::THREADS);
  const dim3 grid((uint32_t)p.ranges * p.all_blocks);
  if (p.ranges > 1) {
    hipError_t e = pg_launch(k_selective_ends<T, LN>, grid, block, 0, L, SelArgs{c, p});
    if (e == hipSuccess) e = selective_groups<LN>(c, p, 1, L);
    if (e != hipSuccess) return e;
  }
  return pg_launch(k_selective<T, LN>, grid, block, 0, L, SelArgs{c, p});
}

template <class T, int LN>
hipError_t step(const SelCall& c, const Launch& L) {
  const int blocks = ceil_div(c.D, kBlock / LN);
  const int64_t grid = std::min<int64_t>((int64_t)c.seqs.nseq * blocks, 1 << 20);
  return pg_launch(k_selective_step<T, LN>, dim3((uint32_t)grid), dim3(kBlock), 0, L, c, blocks);
}

// Channels times ranges of any call of up to D channels: one range, or as many as give
// the workgroups of up to CB channels.
int64_t range_channels(int D, int N) {
  return std::max<int64_t>(D, (int64_t)kSelMostWorkgroups * sel_channels(sel_lanes(N)));
}

}  // namespace

SelRoom selective_room(int64_t tokens, int D, int N) {
  // Fewer states have fewer lanes and wider workgroups: the sizes below grow with N, but for
  // the channels of a workgroup, which are taken at their most.
  SelRoom r;
  const int LN = sel_lanes(N), NP = 4 * LN;
  const int64_t rc = range_channels(D, 1), grouped = rc + rc / kSelGroup + D;
  r.states = (size_t)grouped * NP;
  r.sums = (size_t)grouped;
  r.info = 2 * (size_t)kSelMostWorkgroups;
  r.part_s = 2 * (size_t)rc;
  // blocks of a head's channels, where there are two or more: at most twice D / CB
  r.part_bc = (size_t)tokens * 2 * N * (2 * (size_t)D / sel_channels(LN) + 2);
  return r;
}

hipError_t launch_selective(const SelCall& c, int dtype, SelSpace space, const Launch& L) {
  const SelPlan p = selective_plan(c.seqs, c.D, c.N, c.groups, space);
  return by_format(dtype, [&](auto v) {
    using E = decltype(v);
    return by_lanes(c.N, [&](auto ln) { return forward<E, decltype(ln)::value>(c, p, L); });
  });
}

template <class T>  // in a file for each format
hipError_t selective_grad(const SelCall& c, const SelPlan& p, const Launch& L);

hipError_t launch_selective_grad(const SelCall& c, int dtype, SelSpace space, const Launch& L) {
  const SelPlan p = selective_plan(c.seqs, c.D, c.N, c.groups, space);
  return by_format(dtype, [&](auto v) { return selective_grad<decltype(v)>(c, p, L); });
}

hipError_t launch_selective_step(const SelCall& c, int dtype, const Launch& L) {
  return by_format(dtype, [&](auto v) {
    using E = decltype(v);
    return by_lanes(c.N, [&](auto ln) { return step<E, decltype(ln)::value>(c, L); });
  });
}

}  // namespace pg
