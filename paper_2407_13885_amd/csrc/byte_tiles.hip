// Attention over a paged cache in 8 bits by blocks of 128 rows (paged_tiles.h): scores as they are; and when.
#include "paged_tiles.h"

#include <cstdlib>
#include <cstring>

namespace attnw {

bool prefers_byte_tiles(const PagedArgs& p)
{
    // (ATTNW_PAGED_KERNEL=rows / =tiles: tests and measurements compare the two)
    const char* force = getenv("ATTNW_PAGED_KERNEL");
    if (force && strcmp(force, "rows") == 0) return false;
    if (force && strcmp(force, "tiles") == 0) return true;
    const int64_t group = p.heads / p.cache.kv_heads, rows = p.tokens * group, all = p.tokens * p.heads, d = p.cache.row_bytes;
    if (rows < 48 * (int64_t)p.cache.batch) return false;
    return all * d >= 1 << 19;
}

int64_t byte_tiles_workspace(const PagedArgs& p) { return p.dt == DType::F32 ? byte_tiles_workspace_f32(p) : byte_tiles_workspace<uint16_t>(p); }

hipError_t launch_byte_tiles(const PagedArgs& p, const ScalesView& scales, hipStream_t stream)
{
    if (p.dt == DType::F32) return launch_byte_tiles_f32(p, scales, stream);
    switch (rule_mode(p.rule)) {
    case kPlain: return launch_byte_tiles<uint16_t, kPlain>(p, scales, stream);
    case kCap: return launch_byte_tiles_cap(p, scales, stream);
    case kBias: return launch_byte_tiles_bias(p, scales, stream);
    default: return launch_byte_tiles_both(p, scales, stream);
    }
}

}  // namespace attnw
