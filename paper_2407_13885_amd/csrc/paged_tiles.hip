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
    // Rows / tiles, us, by the rows of a sequence: bf16, 16 sequences of 4096 slots, 8 kv heads of 128: 32 59 / 62, 48 126 / 66, 128 213 / 98, 512 847 / 156; fp32
    // 32 150 / 182, 64 290 / 200, 128 565 / 350.  Few blocks leave workgroups of the larger kind with little each: one sequence of 16384 slots, 8 kv heads, 128 rows
    // 62 / 96, 256 109 / 100, 512 198 / 88; one kv head, 1024 rows 64 / 95.
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
