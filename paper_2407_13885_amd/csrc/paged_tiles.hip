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
    // Small blocks read K and V once for every 16 rows, large ones leave partial results of 128 rows (fp32: 64) to a join: the rows of all kv heads decide, and the head
    // size, with which reading grows faster.  Lengths are not known here.  Small / large, us, one sequence of 4096 slots, of 16384, 8 kv heads:
    // bf16, 256 rows: d = 64 18 / 55, 38 / 61, 128 36 / 89, 102 / 99, 256 96 / 64, 334 / 108; 512 rows: d = 64 23 / 56, 62 / 69, 128 55 / 65, 189 / 87, 256 171 / 75, 645 / 159;
    // 1024 rows: d = 64 39 / 39, 118 / 66, 128 102 / 63, 371 / 107.  With a cap or a bias, 8192 slots: d = 64, 512 rows 41 / 67, 1024 75 / 59; d = 128, 256 rows 63 / 96, 512 106 / 79.
    // fp32, 64 rows: d = 128 30 / 57, 80 / 89, 256 77 / 75, 250 / 156; 256 rows: d = 64 36 / 54, 111 / 125, 128 78 / 75, 272 / 200, 256 248 / 137, 929 / 451.
    // Blocks of few rows: 16 sequences of 4096 slots, d = 128, bf16, 32 rows each 56 / 58, 48 131 / 65; fp32, 32 rows 150 / 182, 64 290 / 200.
    const int64_t group = p.heads / p.cache.kv_heads, rows = p.tokens * group, all = p.tokens * p.heads;
    const int64_t d = p.cache.row_bytes / (p.dt == DType::F32 ? 4 : 2);
    if (rows < 48 * (int64_t)p.cache.batch) return false;
    return p.dt == DType::F32 ? all * d * d >= 3 << 23 : all * d >= 1 << 19;
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
