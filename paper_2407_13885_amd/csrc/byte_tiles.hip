// Attention over a paged cache in 8 bits by blocks of 128 rows (paged_tiles.h): scores as they are; and when a call goes there.
#include "paged_tiles.h"

#include <cstdlib>
#include <cstring>

namespace attnw {

bool prefers_byte_tiles(const PagedArgs& p)
{
    const int64_t group = p.heads / p.cache.kv_heads, rows = p.tokens * group, all = p.tokens * p.heads;
    const bool f32 = p.dt == DType::F32, wide = p.cache.row_bytes > 128;
    // fp32: blocks of 16 rows, whose waves share nothing, are the faster ones up to d = 128 however many there are (512 tokens over 3584 slots, 32 heads on 8: d = 64 76 / 85 us,
    // 128 133 / 133), but for d = 80 and 96, which do not fill their place there (132 / 106).
    // (d = 112 takes there what 128 does, 116 / 116 on another day; large blocks are not built for it.)
    if (f32 && !wide && (p.cache.row_bytes <= 64 || p.cache.row_bytes > 96)) return false;
    // (ATTNW_PAGED_KERNEL=rows / =tiles: tests and measurements compare the two)
    const char* force = getenv("ATTNW_PAGED_KERNEL");
    if (force && strcmp(force, "rows") == 0) return false;
    if (force && strcmp(force, "tiles") == 0) return true;
    // Small blocks read and convert K and V once for every 32 rows (beyond d = 128, and in fp32: 16), large ones leave partial results of 128 rows to a join.
    // Small / large, us, one sequence of 4096 slots, of 16384, 32 heads on 8, bf16:  64 tokens: d = 64 20 / 24, 36 / 32, 128 27 / 32, 50 / 45;  128 tokens: d = 64
    // 26 / 27, 58 / 41, 128 36 / 38, 81 / 60;  256 tokens: d = 64 37 / 32, 100 / 61, 128 50 / 45, 140 / 91;  d = 256, 16 tokens: 28 / 28, 56 / 51, 32 tokens: 38 / 33, 95 / 58.
    // fp32, 16 tokens: d = 160 26 / 26, 52 / 52, 256 30 / 40, 63 / 83;  32 tokens: d = 96 23 / 24, 46 / 39, 160 35 / 30, 89 / 55, 256 42 / 48, 106 / 97;  64 tokens: d = 96 31 / 28,
    // 75 / 61, 256 62 / 63, 188 / 159;  256 tokens: d = 96 70 / 66, 245 / 192, 160 159 / 97, 574 / 295, 256 192 / 170, 689 / 549.
    // Sequences beside each other, 16 of 4096 slots, bf16: d = 64, 64 rows each 36 / 40, 128 rows 55 / 43; d = 128 53 / 65, 78 / 71; d = 256, 32 rows 90 / 145, 64 rows 172 / 148.
    // fp32: d = 96, 64 rows 70 / 86, 128 rows 133 / 107; d = 160, 32 rows 84 / 143, 64 rows 161 / 146.
    if (rows < (wide ? 48 : f32 ? 128 : 96) * (int64_t)p.cache.batch) return false;
    return wide ? all >= (f32 ? 1024 : 768) : f32 ? all >= 2048 : all > 2048;
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
