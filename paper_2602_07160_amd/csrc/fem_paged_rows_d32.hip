// Few-row paged reads at d_qk = 32 (fem_paged_rows.h).

#include "fem_paged_launch.h"

namespace fem {

template hipError_t paged_rows<32, 32>(const PagedArgs&, const ReadArgs&, const PagedPlan&, int,
                                         hipStream_t);

}  // namespace fem
