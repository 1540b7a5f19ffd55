// Launches of the paged read of one pair of widths.
#pragma once

#include "fem_paged_wide.h"

#include <algorithm>
#include <type_traits>

namespace fem {

template <int DK, int DV>
hipError_t paged_rows(const PagedArgs& a, const ReadArgs& r, const PagedPlan& plan, int kv,
                      hipStream_t stream) {
  const dim3 grid((unsigned)plan.groups), block(kRowThreads);
  auto go = [&](auto kernel) { hipLaunchKernelGGL(kernel, grid, block, 0, stream, a, r); };
  auto pick = [&](auto rb) {
    constexpr int RB = decltype(rb)::value;
    if (kv == FEM_KV_BF16) go(paged_rows_kernel<DK, DV, FEM_KV_BF16, RB>);
    else if (kv == FEM_KV_E4M3) go(paged_rows_kernel<DK, DV, FEM_KV_E4M3, RB>);
    else go(paged_rows_kernel<DK, DV, FEM_KV_INT8, RB>);
  };
  if (plan.rps <= 16) pick(std::integral_constant<int, 1>());
  else pick(std::integral_constant<int, 2>());
  hipError_t e = hipGetLastError();
  if (e != hipSuccess || plan.target == 0) return e;
  const Work w{r.G, kRowsMax, kRowTile, 0, r.most_rows, a.max_q, r.causal != 0};
  // (only calls with at most `target` row blocks of all heads are split)
  const size_t blocks = std::min<size_t>((size_t)plan.row_blocks * a.heads, plan.target);
  const int chunks = (r.rps + kMergeRows - 1) / kMergeRows;
  hipLaunchKernelGGL((paged_merge_kernel<DV, kMergeRows>), dim3((unsigned)(blocks * chunks)),
                     dim3(kMergeThreads), 0, stream, a, r, w, r.tps, r.part, r.rps);
  return hipGetLastError();
}

template <int DK, int DV>
hipError_t paged_wide(const PagedArgs& a, const ReadArgs& r, const PagedPlan& plan, int kv,
                      hipStream_t stream) {
  const size_t most = (size_t)plan.wide_blocks * a.heads;  // row blocks at most
  const size_t pieces = r.split_wide ? std::max<size_t>(most, kWideGroups * kWideRounds) : most;
  const dim3 grid((unsigned)std::min<size_t>(pieces, kWideGroups)), block(512);
  auto go = [&](auto kernel) { hipLaunchKernelGGL(kernel, grid, block, 0, stream, a, r); };
  if (kv == FEM_KV_BF16) go(paged_wide_kernel<DK, DV, FEM_KV_BF16>);
  else if (kv == FEM_KV_E4M3) go(paged_wide_kernel<DK, DV, FEM_KV_E4M3>);
  else go(paged_wide_kernel<DK, DV, FEM_KV_INT8>);
  hipError_t e = hipGetLastError();
  if (e != hipSuccess || !r.split_wide) return e;
  const Work w{r.G, kWideRows, kWideTile, r.wide_least, 1ll << 60, a.max_q, r.causal != 0};
  // (only calls of at most this many row blocks are split)
  const size_t blocks = std::min<size_t>(most, (size_t)kWideGroups * kWideRounds);
  const int chunks = (r.wide_rps + kWideMergeRows - 1) / kWideMergeRows;
  hipLaunchKernelGGL((paged_merge_kernel<DV, kWideMergeRows>), dim3((unsigned)(blocks * chunks)),
                     dim3(kMergeThreads), 0, stream, a, r, w, r.tps + 1, r.wide_part, r.wide_rps);
  return hipGetLastError();
}

}  // namespace fem
