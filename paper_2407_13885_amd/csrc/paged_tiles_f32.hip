// Attention over a paged cache by blocks of 64 rows (paged_tiles.h), fp32.
#include "paged_tiles.h"

namespace attnw {

int64_t paged_tiles_workspace_f32(const PagedArgs& p) { return tiles_workspace<float>(p); }

hipError_t launch_paged_tiles_f32(const PagedArgs& p, hipStream_t stream)
{
    switch (rule_mode(p.rule)) {
    case kPlain: return launch_tiles<float, kPlain>(p, stream);
    case kCap: return launch_tiles<float, kCap>(p, stream);
    case kBias: return launch_tiles<float, kBias>(p, stream);
    default: return launch_tiles<float, kCap | kBias>(p, stream);
    }
}

}  // namespace attnw
