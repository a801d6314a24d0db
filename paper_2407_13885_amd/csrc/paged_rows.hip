// Attention over a paged cache by blocks of 16 rows (paged_rows.h), bf16; and which kernel a call goes to.
#include "paged_rows.h"

namespace attnw {

int64_t paged_workspace(const PagedArgs& p)
{
    return p.dt == DType::F32 ? paged_rows_workspace_f32(p) : prefers_paged_tiles(p) ? paged_tiles_workspace(p) : rows_workspace<uint16_t>(p);
}

hipError_t launch_paged_attention(const PagedArgs& p, hipStream_t stream)
{
    return p.dt == DType::F32 ? launch_paged_rows_f32(p, stream) : prefers_paged_tiles(p) ? launch_paged_tiles(p, stream) : launch_rows<uint16_t>(p, stream);
}

}  // namespace attnw
