// Launch of the few-row paged read of one pair of widths.
#pragma once

#include "fem_paged_rows.h"

namespace fem {

template <int DK, int DV>
hipError_t paged_rows(const PagedArgs& a, const ReadArgs& r, const PagedPlan& plan, int kv,
                      hipStream_t stream) {
  const dim3 grid((unsigned)plan.slots), block(kRowThreads);
  auto go = [&](auto kernel) { hipLaunchKernelGGL(kernel, grid, block, 0, stream, a, r); };
  if (kv == FEM_KV_BF16) go(paged_rows_kernel<DK, DV, FEM_KV_BF16>);
  else if (kv == FEM_KV_E4M3) go(paged_rows_kernel<DK, DV, FEM_KV_E4M3>);
  else go(paged_rows_kernel<DK, DV, FEM_KV_INT8>);
  const hipError_t e = hipGetLastError();
  if (e != hipSuccess || plan.target == 0) return e;
  hipLaunchKernelGGL((paged_merge_kernel<DV>), dim3((unsigned)(plan.row_blocks * a.heads)),
                     dim3(kMergeThreads), 0, stream, a, r);
  return hipGetLastError();
}

}  // namespace fem
