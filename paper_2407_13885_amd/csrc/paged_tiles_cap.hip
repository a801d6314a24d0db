// Attention over a paged cache by blocks of 128 rows (paged_tiles.h): capped scores.
#include "paged_tiles.h"

namespace attnw {

hipError_t launch_paged_tiles_cap(const PagedArgs& p, hipStream_t stream) { return launch_tiles<uint16_t, kCap>(p, stream); }

}  // namespace attnw
