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
    // bf16, 256 rows: d = 64 18 / 22, 38 / 29, 128 35 / 32, 103 / 45, 256 97 / 38, 338 / 87; 512 rows: d = 64 22 / 24, 61 / 38, 128 54 / 35, 189 / 58, 256 173 / 75, 650 / 167;
    // 1024 rows: d = 64 38 / 28, 116 / 57, 128 103 / 42, 372 / 88.  With a cap, 8192 slots: d = 64, 512 rows 40 / 33, 1024 74 / 48; d = 128, 256 rows 63 / 38, 512 108 / 46.
    // fp32, 64 rows: d = 128 31 / 31, 80 / 65, 256 78 / 49, 254 / 134; 256 rows: d = 64 36 / 39, 113 / 111, 128 79 / 60, 273 / 188, 256 249 / 137, 934 / 453.
    // Blocks of few rows: 16 sequences of 4096 slots, d = 128, bf16, 32 rows each 58 / 72, 48 132 / 74; fp32, 32 rows 145 / 188, 64 285 / 199.
    // (The bounds are from when a join took 40 us of a call by large blocks; it takes 4 to 10 now, and in bf16 they could lie at half of what they are.  They stand, so
    // that a call goes on giving the results it gave.)
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
