// Launches of the dropout and the scores.
#include "operators.h"

#include <algorithm>

#include "dropout_dev.h"
#include "logits_dev.h"

namespace pg {

hipError_t launch_dropout(const DropoutCall& c, const Launch& L) {
  const int64_t total = c.a.rows * ((c.a.d + 7) / 8);
  const int grid = (int)std::min<int64_t>((total + kBlock - 1) / kBlock, 16 * kCus);
  return by_format(c.a.dtype, [&](auto v) {
    return pg_launch(k_dropout<decltype(v)>, dim3(grid), dim3(kBlock), 0, L, c);
  });
}

hipError_t launch_logits(const LogitsCall& c, const Launch& L) {
  return by_format(c.a.dtype, [&](auto v) {
    return pg_launch(k_logits<decltype(v)>, dim3(c.a.rows), dim3(kBlock), 0, L, c);
  });
}

}  // namespace pg
