// Paged reads of many rows, d_qk = 64, d_v = 64.

#include "fem_paged_launch.h"

namespace fem {
template hipError_t paged_wide<64, 64>(const PagedArgs&, const ReadArgs&, const PagedPlan&, int,
                                     hipStream_t);
}  // namespace fem
