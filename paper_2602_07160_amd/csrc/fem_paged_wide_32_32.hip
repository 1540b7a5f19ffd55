// Paged reads of many rows, d_qk = 32, d_v = 32.

#include "fem_paged_launch.h"

namespace fem {
template hipError_t paged_wide<32, 32>(const PagedArgs&, const ReadArgs&, const PagedPlan&, int,
                                     hipStream_t);
}  // namespace fem
