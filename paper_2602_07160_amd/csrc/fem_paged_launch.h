// Launches of the paged read of one pair of widths.
#pragma once

#include "fem_paged_wide.h"

#include <algorithm>
#include <type_traits>

namespace fem {

template <int DK, int DV>
hipError_t paged_rows(const PagedArgs& a, const ReadArgs& r, const PagedPlan& plan, int kv,
                      hipStream_t stream) {
  const dim3 grid((unsigned)plan.groups), block(64 * plan.waves);
  auto go = [&](auto kernel) { hipLaunchKernelGGL(kernel, grid, block, 0, stream, a, r); };
  auto pick = [&](auto rb, auto nw) {
    constexpr int RB = decltype(rb)::value, NW = decltype(nw)::value;
    if (kv == FEM_KV_BF16) go(paged_rows_kernel<DK, DV, FEM_KV_BF16, RB, NW>);
    else if (kv == FEM_KV_E4M3) go(paged_rows_kernel<DK, DV, FEM_KV_E4M3, RB, NW>);
    else go(paged_rows_kernel<DK, DV, FEM_KV_INT8, RB, NW>);
  };
  const std::integral_constant<int, 1> one;
  const std::integral_constant<int, 2> two;
  const std::integral_constant<int, kRowWaves> few;
  const std::integral_constant<int, 2 * kRowWaves> many;
  if (plan.waves == kRowWaves) {
    if (plan.rps <= 16) pick(one, few);
    else pick(two, few);
  } else {
    if (plan.rps <= 16) pick(one, many);
    else pick(two, many);
  }
  return hipGetLastError();
}

template <int DK, int DV>
hipError_t paged_wide(const PagedArgs& a, const ReadArgs& r, const PagedPlan& plan, int kv,
                      hipStream_t stream) {
  const dim3 grid((unsigned)plan.wide_groups), block(512);
  auto go = [&](auto kernel) { hipLaunchKernelGGL(kernel, grid, block, 0, stream, a, r); };
  if (kv == FEM_KV_BF16) go(paged_wide_kernel<DK, DV, FEM_KV_BF16>);
  else if (kv == FEM_KV_E4M3) go(paged_wide_kernel<DK, DV, FEM_KV_E4M3>);
  else go(paged_wide_kernel<DK, DV, FEM_KV_INT8>);
  return hipGetLastError();
}

}  // namespace fem
