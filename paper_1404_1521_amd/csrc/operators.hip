// Launches of the dropout and the scores.
#include "operators.h"

#include <algorithm>

#include "dropout_dev.h"
#include "logits_dev.h"

namespace pg {

namespace {

template <class T, int U>
hipError_t dropout_of(const DropoutCall& c, int64_t total, const Launch& L) {
  static_assert(U * kBlock <= kDropPlaces, "places of a workgroup");
  const int64_t grid = (total + kBlock * U - 1) / (kBlock * U);
  if (grid > INT32_MAX) return hipErrorInvalidValue;
  auto k = c.a.ids ? (c.a.add ? k_dropout<T, true, true, U> : k_dropout<T, false, true, U>)
                   : (c.a.add ? k_dropout<T, true, false, U> : k_dropout<T, false, false, U>);
  return pg_launch(k, dim3((uint32_t)grid), dim3(kBlock), 0, L, c);
}

}  // namespace

hipError_t launch_dropout(const DropoutCall& c, const Launch& L) {
  const int64_t total = c.a.rows * c.groups;
  return by_format(c.a.dtype, [&](auto v) {
    using T = decltype(v);
    return total >= (int64_t)4 * kBlock * 4 * kCus ? dropout_of<T, 4>(c, total, L)
                                                   : dropout_of<T, 1>(c, total, L);
  });
}

hipError_t launch_logits(LogitsCall c, const Launch& L) {
  // Long parts read the history and the row's rules fewer times; short ones spread a few
  // rows over the chip.  The longest that give every CU two workgroups: 256 rows of
  // 1,000,000 in parts of 2,048 words 456 us, 4,096 328, 8,192 266, 16,384 (fewer
  // workgroups to a CU) 276; 48 rows of 32,003 in parts of 1,024 9.8, 2,048 9.2, 4,096
  // 10.2.
  int E = 32;
  while (E > 4 && (int64_t)c.a.rows * ceil_div(c.a.V, E * kBlock) < 2 * kCus) E /= 2;
  c.tiles = ceil_div(c.a.V, E * kBlock);
  if ((int64_t)c.a.rows * c.tiles > INT32_MAX) return hipErrorInvalidValue;
  return by_format(c.a.dtype, [&](auto v) {
    using T = decltype(v);
    const bool many = c.a.history && c.a.history_cap > 32767;
    auto k = E == 32   ? (many ? k_logits<T, 32, true> : k_logits<T, 32, false>)
             : E == 16 ? (many ? k_logits<T, 16, true> : k_logits<T, 16, false>)
             : E == 8  ? (many ? k_logits<T, 8, true> : k_logits<T, 8, false>)
                       : (many ? k_logits<T, 4, true> : k_logits<T, 4, false>);
    return pg_launch(k, dim3(c.a.rows * c.tiles), dim3(kBlock), 0, L, c);
  });
}

}  // namespace pg
