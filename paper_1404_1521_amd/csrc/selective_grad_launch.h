// Launches of the selective scan's gradient, in one format: each is compiled by itself.
#pragma once
#include "selective_grad_dev.h"
#include "selective_plan.h"

namespace pg {

template <class T, int LN>
hipError_t grad_of_lanes(const SelCall& c, const SelPlan& p, const Launch& L) {
  const dim3 grid((uint32_t)p.ranges * p.all_blocks), block(SelShape<LN>::THREADS);
  hipError_t e = hipSuccess;
  if (p.ranges > 1) e = pg_launch(k_selective_grad_ends<T, LN>, grid, block, 0, L, SelArgs{c, p});
  if (e == hipSuccess) e = selective_groups<LN>(c, p, -1, L);
  if (e == hipSuccess) e = pg_launch(k_selective_grad<T, LN>, grid, block, 0, L, SelArgs{c, p});
  if (e != hipSuccess) return e;
  const int params = (int)(((int64_t)c.D * (c.N + 2) + kSumOutputs - 1) / kSumOutputs);
  const int64_t rest = p.blocks == 1 ? 0 : (int64_t)c.groups * 2 * c.N * c.seqs.tokens;
  const int sums = (int)std::min<int64_t>((rest + kBlock - 1) / kBlock, 16 * kCus);
  return pg_launch(k_selective_sums<T>, dim3(params + sums), dim3(kBlock), 0, L, c, p, 4 * LN, params);
}

template <class T>
hipError_t selective_grad(const SelCall& c, const SelPlan& p, const Launch& L) {
  return by_lanes(c.N, [&](auto ln) { return grad_of_lanes<T, decltype(ln)::value>(c, p, L); });
}

}  // namespace pg
