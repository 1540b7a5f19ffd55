// Few-row paged reads at d_qk = 64 (fem_paged_rows.h).

#include "fem_paged_launch.h"

namespace fem {

template hipError_t paged_rows<64, 64>(const PagedArgs&, const ReadArgs&, const PagedPlan&, int,
                                         hipStream_t);
template hipError_t paged_rows<64, 32>(const PagedArgs&, const ReadArgs&, const PagedPlan&, int,
                                         hipStream_t);

}  // namespace fem
