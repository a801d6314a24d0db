// Attention over a paged cache by blocks of 128 rows (paged_tiles.h): scores as they are; and when.
#include "paged_tiles.h"

#include <cstdlib>
#include <cstring>

namespace attnw {

bool prefers_paged_tiles(const PagedArgs& p)
{
    // (ATTNW_PAGED_KERNEL=rows / =tiles: tests and measurements compare the two)
    const char* force = getenv("ATTNW_PAGED_KERNEL");
    if (force && strcmp(force, "rows") == 0) return false;
    if (force && strcmp(force, "tiles") == 0) return true;
    const int64_t group = p.heads / p.cache.kv_heads, rows = p.tokens * group, batch = p.cache.batch;
    const int64_t block = p.dt == DType::F32 ? 64 : 128, blocks = (rows / block + batch) * p.cache.kv_heads;
    return rows >= 48 * batch && blocks >= 48;
}

int64_t paged_tiles_workspace(const PagedArgs& p) { return p.dt == DType::F32 ? paged_tiles_workspace_f32(p) : tiles_workspace<uint16_t>(p); }

hipError_t launch_paged_tiles(const PagedArgs& p, hipStream_t stream)
{
    if (p.dt == DType::F32) return launch_paged_tiles_f32(p, stream);
    switch (rule_mode(p.rule)) {
    case kPlain: return launch_tiles<uint16_t, kPlain>(p, stream);
    case kCap: return launch_paged_tiles_cap(p, stream);
    case kBias: return launch_paged_tiles_bias(p, stream);
    default: return launch_paged_tiles_both(p, stream);
    }
}

}  // namespace attnw
