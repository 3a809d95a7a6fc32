// Launches of the beams' selection and of the reordering.
#include "operators.h"

#include <algorithm>

#include "beam_dev.h"

namespace pg {

hipError_t launch_beam(BeamCall c, int dtype, const Launch& L) {
  // As many parts as give every CU two workgroups, of at least 1,024 words.
  const int64_t rows = (int64_t)c.groups * c.beams;
  const int64_t want = std::max<int64_t>(1, (2 * kCus + rows - 1) / rows);
  const int64_t units = ((int64_t)c.V + kBeamMinPart - 1) / kBeamMinPart, each = (units + want - 1) / want;
  c.part_words = (int)(each * kBeamMinPart);
  c.parts = (int)((units + each - 1) / each);
  const hipError_t e = by_format(dtype, [&](auto v) {
    return pg_launch(k_beam_parts<decltype(v)>, dim3((uint32_t)(rows * c.parts)), dim3(kBlock), 0, L, c);
  });
  if (e != hipSuccess) return e;
  return pg_launch(k_beam_join, dim3(c.groups), dim3(kBlock), 0, L, c);
}

hipError_t launch_reorder(const ReorderCall& c, const Launch& L) {
  const int64_t all = c.first[c.count];
  if (all == 0) return hipSuccess;
  return pg_launch(k_reorder, dim3((uint32_t)std::min<int64_t>(all, 1 << 22)), dim3(kBlock), 0, L, c);
}

}  // namespace pg
