// Attention over a paged cache by blocks of 16 rows (paged_rows.h), fp32.
#include "paged_rows.h"

namespace attnw {

int64_t paged_rows_workspace_f32(const PagedArgs& p) { return rows_workspace<float>(p); }
hipError_t launch_paged_rows_f32(const PagedArgs& p, hipStream_t stream) { return launch_rows<float>(p, stream); }

}  // namespace attnw
