// Launches of the beams' selection and of the reordering.
#include "operators.h"

#include <algorithm>

#include "beam_dev.h"

namespace pg {

namespace {

constexpr int kJoinEach = 8;  // keys of a thread in a batch of the join

template <class T>
hipError_t parts_of(const BeamCall& c, int E, const Launch& L) {
  auto k = E == 64 ? k_beam_parts<T, 64> : E == 32 ? k_beam_parts<T, 32> : E == 16 ? k_beam_parts<T, 16>
         : E == 8  ? k_beam_parts<T, 8>  : k_beam_parts<T, 4>;
  return pg_launch(k, dim3((uint32_t)(c.groups * c.beams * c.parts)), dim3(kBlock), 0, L, c);
}

}  // namespace

hipError_t launch_beam(BeamCall c, int dtype, const Launch& L) {
  // Long parts are fewer picks to find and to join; short ones spread a few rows over the chip:
  // the longest that still give two workgroups to a CU.  (One to a CU is alike, but for 64
  // picks, 33 us for 36 in 32 x 8 rows of 32,000; four cost 61 there and give nothing elsewhere.)
  int E = 64;
  const int64_t rows = (int64_t)c.groups * c.beams;
  while (E > 4 && rows * ceil_div(c.V, E * kBlock) < 2 * kCus) E /= 2;
  c.parts = ceil_div(c.V, E * kBlock);
  const hipError_t e = by_format(dtype, [&](auto v) { return parts_of<decltype(v)>(c, E, L); });
  if (e != hipSuccess) return e;
  return pg_launch(k_beam_join<kJoinEach>, dim3(c.groups), dim3(kBlock), 0, L, c);
}

hipError_t launch_reorder(const ReorderCall& c, const Launch& L) {
  const int64_t all = c.first[c.count];
  if (all == 0) return hipSuccess;
  return pg_launch(k_reorder, dim3((uint32_t)std::min<int64_t>(all, 1 << 22)), dim3(kBlock), 0, L, c);
}

}  // namespace pg
