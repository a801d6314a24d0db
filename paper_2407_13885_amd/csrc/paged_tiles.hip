// Attention over a paged cache by blocks of 128 rows (paged_tiles.h): scores as they are; and when.
#include "paged_tiles.h"

#include <cstdlib>
#include <cstring>

namespace attnw {

bool prefers_paged_tiles(const PagedArgs& p)
{
    if (p.dt != DType::BF16) return false;
    // (ATTNW_PAGED_KERNEL=rows / =tiles: tests and measurements compare the two)
    const char* force = getenv("ATTNW_PAGED_KERNEL");
    if (force && strcmp(force, "rows") == 0) return false;
    if (force && strcmp(force, "tiles") == 0) return true;
    const int64_t rows = p.tokens * (p.heads / p.cache.kv_heads);
    return rows > 48 * (int64_t)p.cache.batch;
}

int64_t paged_tiles_workspace(const PagedArgs& p)
{
    return by_row(p.cache.row_bytes, [&](auto ub) { return partial_bytes(workgroups<decltype(ub)::value>(), TilesCfg<decltype(ub)::value>::ROWS, TilesCfg<decltype(ub)::value>::COLS); });
}

hipError_t launch_paged_tiles(const PagedArgs& p, hipStream_t stream)
{
    switch (rule_mode(p.rule)) {
    case kPlain: return launch_tiles<kPlain>(p, stream);
    case kCap: return launch_paged_tiles_cap(p, stream);
    case kBias: return launch_paged_tiles_bias(p, stream);
    default: return launch_paged_tiles_both(p, stream);
    }
}

}  // namespace attnw
