// Attention over a paged cache in 8 bits by blocks of 16 rows (byte_rows.h), fp32.
#include "byte_rows.h"

namespace attnw {

int64_t byte_rows_workspace_f32(const PagedArgs& p) { return rows_workspace<float>(p); }

hipError_t launch_byte_rows_f32(const PagedArgs& p, const ScalesView& scales, hipStream_t stream) { return launch_rows<float>(p, scales, stream); }

}  // namespace attnw
