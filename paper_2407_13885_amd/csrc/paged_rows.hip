// Attention over a paged cache by blocks of 16 rows (paged_rows.h), bf16; and which kernel a call goes to.
#include "paged_rows.h"

namespace attnw {

int64_t paged_workspace(const PagedArgs& p)
{
    return prefers_paged_tiles(p) ? paged_tiles_workspace(p) : p.dt == DType::F32 ? paged_rows_workspace_f32(p) : rows_workspace<uint16_t>(p);
}

hipError_t launch_paged_attention(const PagedArgs& p, hipStream_t stream)
{
    return prefers_paged_tiles(p) ? launch_paged_tiles(p, stream) : p.dt == DType::F32 ? launch_paged_rows_f32(p, stream) : launch_rows<uint16_t>(p, stream);
}

}  // namespace attnw
