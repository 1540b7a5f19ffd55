// Paged reads of few rows, d_qk = 64, d_v = 32.

#include "fem_paged_launch.h"

namespace fem {
template hipError_t paged_rows<64, 32>(const PagedArgs&, const ReadArgs&, const PagedPlan&, int,
                                     hipStream_t);
}  // namespace fem
