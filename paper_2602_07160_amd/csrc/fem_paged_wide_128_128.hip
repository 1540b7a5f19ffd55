// Paged reads of many rows, d_qk = 128, d_v = 128.

#include "fem_paged_launch.h"

namespace fem {
template hipError_t paged_wide<128, 128>(const PagedArgs&, const ReadArgs&, const PagedPlan&, int,
                                     hipStream_t);
}  // namespace fem
