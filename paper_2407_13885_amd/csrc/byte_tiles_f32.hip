// Attention over a paged cache in 8 bits by blocks of 128 rows (paged_tiles.h), fp32, d = 80, 96 and above 128.
#include "paged_tiles.h"

namespace attnw {

int64_t byte_tiles_workspace_f32(const PagedArgs& p) { return byte_tiles_workspace<float>(p); }

hipError_t launch_byte_tiles_f32(const PagedArgs& p, const ScalesView& scales, hipStream_t stream)
{
    switch (rule_mode(p.rule)) {
    case kPlain: return launch_byte_tiles<float, kPlain>(p, scales, stream);
    case kCap: return launch_byte_tiles<float, kCap>(p, scales, stream);
    case kBias: return launch_byte_tiles<float, kBias>(p, scales, stream);
    default: return launch_byte_tiles<float, kCap | kBias>(p, scales, stream);
    }
}

}  // namespace attnw
