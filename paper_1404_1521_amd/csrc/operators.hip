// Launches of the sequence operators' kernels.
#include "operators.h"

#include <algorithm>

#include "dropout_dev.h"
#include "logits_dev.h"
#include "recurrence_dev.h"

namespace pg {

namespace {

// Calls f with a value of the storage type `dtype` (POLYGLOT_F32, _BF16, _F16).
template <class F>
hipError_t by_format(int dtype, F f) {
  if (dtype == POLYGLOT_F32) return f(float{});
  if (dtype == POLYGLOT_BF16) return f(BF16{});
  return f(F16{});
}

}  // namespace

hipError_t launch_dropout(const DropoutCall& c, const Launch& L) {
  const int64_t total = c.a.rows * ((c.a.d + 7) / 8);
  const int grid = (int)std::min<int64_t>((total + kBlock - 1) / kBlock, 16 * kCus);
  return by_format(c.a.dtype, [&](auto v) {
    return pg_launch(k_dropout<decltype(v)>, dim3(grid), dim3(kBlock), 0, L, c);
  });
}

hipError_t launch_recurrence(const RecCall& c, int dtype, int form, bool grad, const Launch& L) {
  const int width = c.group > 1 ? kBlock / c.group * c.group : kBlock;
  const dim3 grid(c.nseq, ceil_div(c.D, width));
  return by_format(dtype, [&](auto v) {
    using T = decltype(v);
    constexpr int raw = POLYGLOT_GATE_RAW, sig = POLYGLOT_GATE_SIGMOID;
    auto k = form == raw ? (grad ? k_recurrence<T, raw, true> : k_recurrence<T, raw, false>)
                         : (grad ? k_recurrence<T, sig, true> : k_recurrence<T, sig, false>);
    return pg_launch(k, grid, dim3(kBlock), 0, L, c);
  });
}

hipError_t launch_logits(const LogitsCall& c, const Launch& L) {
  return by_format(c.a.dtype, [&](auto v) {
    return pg_launch(k_logits<decltype(v)>, dim3(c.a.rows), dim3(kBlock), 0, L, c);
  });
}

}  // namespace pg
