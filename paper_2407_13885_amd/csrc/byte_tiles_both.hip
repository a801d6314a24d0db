// Attention over a paged cache in 8 bits by blocks of 128 rows (paged_tiles.h): capped scores with a bias by distance.
#include "paged_tiles.h"

namespace attnw {

hipError_t launch_byte_tiles_both(const PagedArgs& p, const ScalesView& scales, hipStream_t stream) { return launch_byte_tiles<uint16_t, kCap | kBias>(p, scales, stream); }

}  // namespace attnw
