// Launches of the short causal convolution and its gradient.
#include "operators.h"

#include <algorithm>
#include <type_traits>

#include "convolution_dev.h"

namespace pg {

namespace {

// Channels of a thread: 16 bytes in one access; the gradient, which keeps three values a tap
// and channel, takes four.
constexpr int channels(size_t size, bool grad) { return size == 2 && !grad ? 8 : 4; }

// As few lanes as hold all channels; chunks of whole steps.
void cut(ConvCall& c, int V, int workgroups) {
  int log2 = 3;
  while (log2 < 6 && (V << log2) < c.D) ++log2;
  c.lanes_log2 = log2;
  c.blocks = ceil_div(c.D, V << log2);
  const int rows = kBlock >> log2;  // chunks of a workgroup
  const int64_t steps = std::max<int64_t>(1, ((int64_t)c.seqs.tokens + kConvStep - 1) / kConvStep);
  const int64_t want = std::max(1, workgroups / c.blocks) * (int64_t)rows;
  const int64_t each = (steps + want - 1) / want;
  c.chunk = (int)(each * kConvStep);
  c.groups = (int)(((steps + each - 1) / each + rows - 1) / rows);
}

template <class F>
hipError_t by_taps(int K, F f) {
  switch (K) {
    case 1: return f(std::integral_constant<int, 1>{});
    case 2: return f(std::integral_constant<int, 2>{});
    case 3: return f(std::integral_constant<int, 3>{});
    default: return f(std::integral_constant<int, 4>{});
  }
}

}  // namespace

size_t convolution_room(int D) {  // groups, rounded up, times the channels of a row of blocks
  return (size_t)(kConvMaxK + 1) * ((size_t)D + (size_t)(kConvWorkgroups + 1) * 4 * kWave);
}

hipError_t launch_convolution(ConvCall c, int K, int dtype, const Launch& L) {
  return by_format(dtype, [&](auto v) {
    using T = decltype(v);
    return by_taps(K, [&](auto k) {
      constexpr int V = channels(sizeof(T), false);
      cut(c, V, kConvWorkgroups);
      return pg_launch(k_convolution<T, decltype(k)::value, V>, dim3((uint32_t)(c.groups * c.blocks)),
                       dim3(kBlock), 0, L, c);
    });
  });
}

hipError_t launch_convolution_step(ConvCall c, int K, int dtype, const Launch& L) {
  return by_format(dtype, [&](auto v) {
    using T = decltype(v);
    return by_taps(K, [&](auto k) {
      constexpr int V = 4;  // a step's time is latency: more threads, shorter ones
      const int64_t all = (int64_t)c.seqs.nseq * ceil_div(c.D, V);
      const int grid = (int)std::min<int64_t>((all + kBlock - 1) / kBlock, 16 * kCus);
      return pg_launch(k_convolution_step<T, decltype(k)::value, V>, dim3(grid), dim3(kBlock), 0, L, c);
    });
  });
}

hipError_t launch_convolution_grad(ConvCall c, int K, int dtype, const Launch& L) {
  cut(c, channels(4, true), kCus * conv_grad_waves(dtype == POLYGLOT_F32 ? 4 : 2));
  hipError_t e = by_format(dtype, [&](auto v) {
    using T = decltype(v);
    return by_taps(K, [&](auto k) {
      constexpr int V = channels(sizeof(T), true);
      return pg_launch(k_convolution_grad<T, decltype(k)::value, V>, dim3((uint32_t)(c.groups * c.blocks)),
                       dim3(kBlock), 0, L, c);
    });
  });
  if (e != hipSuccess) return e;
  const int64_t all = (int64_t)(K + 1) * c.D;
  return pg_launch(k_convolution_sums, dim3((uint32_t)((all + kSumOutputs - 1) / kSumOutputs)), dim3(kBlock),
                   0, L, c, K);
}

}  // namespace pg
