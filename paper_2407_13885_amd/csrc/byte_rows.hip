// Attention over a paged cache in 8 bits by blocks of 16 rows (byte_rows.h), bf16; and which kernel a call goes to.
#include "byte_rows.h"

namespace attnw {

int64_t byte_workspace(const PagedArgs& p) { return prefers_byte_tiles(p) ? byte_tiles_workspace(p) : p.dt == DType::F32 ? byte_rows_workspace_f32(p) : rows_workspace<uint16_t>(p); }

hipError_t launch_byte_attention(const PagedArgs& p, const ScalesView& scales, hipStream_t stream)
{
    if (prefers_byte_tiles(p)) return launch_byte_tiles(p, scales, stream);
    return p.dt == DType::F32 ? launch_byte_rows_f32(p, scales, stream) : launch_rows<uint16_t>(p, scales, stream);
}

}  // namespace attnw
