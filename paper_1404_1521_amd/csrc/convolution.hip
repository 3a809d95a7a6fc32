// Launches of the short causal convolution and its gradient.
#include "operators.h"

#include <algorithm>
#include <type_traits>

#include "convolution_dev.h"

namespace pg {

namespace {

// As few lanes as hold all channels, four to a lane.
void cut(ConvCall& c) {
  int log2 = 3;
  while (log2 < 6 && (4 << log2) < c.D) ++log2;
  static_assert(1 << 3 == kConvMinLanes, "cut");
  c.lanes_log2 = log2;
  c.blocks = ceil_div(c.D, 4 << log2);
  const int tokens = (kBlock >> log2) * kConvRun;
  c.tiles = std::max(1, ceil_div(c.seqs.tokens, tokens));
  c.groups = std::min(c.tiles, std::max(1, kConvWorkgroups / c.blocks));
}

template <class F>
hipError_t by_taps(int K, F f) {
  switch (K) {
    case 1: return f(std::integral_constant<int, 1>{});
    case 2: return f(std::integral_constant<int, 2>{});
    case 3: return f(std::integral_constant<int, 3>{});
    case 4: return f(std::integral_constant<int, 4>{});
    case 5: return f(std::integral_constant<int, 5>{});
    case 6: return f(std::integral_constant<int, 6>{});
    case 7: return f(std::integral_constant<int, 7>{});
    default: return f(std::integral_constant<int, 8>{});
  }
}

}  // namespace

size_t convolution_room(int D) {
  return (size_t)(kConvMaxK + 1) * std::max<size_t>(D, (size_t)kConvWorkgroups * 4 * kWave);
}

hipError_t launch_convolution(ConvCall c, int K, int dtype, const Launch& L) {
  cut(c);
  return by_format(dtype, [&](auto v) {
    using T = decltype(v);
    return by_taps(K, [&](auto k) {
      return pg_launch(k_convolution<T, decltype(k)::value>, dim3((uint32_t)(c.tiles * c.blocks)), dim3(kBlock),
                       0, L, c);
    });
  });
}

hipError_t launch_convolution_step(ConvCall c, int K, int dtype, const Launch& L) {
  cut(c);
  const int64_t all = (int64_t)c.seqs.nseq * ceil_div(c.D, 4);
  const int grid = (int)std::min<int64_t>((all + kBlock - 1) / kBlock, 16 * kCus);
  return by_format(dtype, [&](auto v) {
    using T = decltype(v);
    return by_taps(K, [&](auto k) {
      return pg_launch(k_convolution_step<T, decltype(k)::value>, dim3(grid), dim3(kBlock), 0, L, c);
    });
  });
}

hipError_t launch_convolution_grad(ConvCall c, int K, int dtype, const Launch& L) {
  cut(c);
  hipError_t e = by_format(dtype, [&](auto v) {
    using T = decltype(v);
    return by_taps(K, [&](auto k) {
      return pg_launch(k_convolution_grad<T, decltype(k)::value>, dim3((uint32_t)(c.groups * c.blocks)),
                       dim3(kBlock), 0, L, c);
    });
  });
  if (e != hipSuccess) return e;
  const int64_t all = (int64_t)(K + 1) * c.D;
  return pg_launch(k_convolution_sums, dim3((uint32_t)((all + kWave - 1) / kWave)), dim3(kBlock), 0, L, c, K);
}

}  // namespace pg
