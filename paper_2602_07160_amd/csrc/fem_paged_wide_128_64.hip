// Paged reads of many rows, d_qk = 128, d_v = 64.

#include "fem_paged_launch.h"

namespace fem {
template hipError_t paged_wide<128, 64>(const PagedArgs&, const ReadArgs&, const PagedPlan&, int,
                                     hipStream_t);
}  // namespace fem
