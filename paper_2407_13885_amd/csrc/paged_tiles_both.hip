// Attention over a paged cache by blocks of 128 rows (paged_tiles.h): capped scores with a bias by distance.
#include "paged_tiles.h"

namespace attnw {

hipError_t launch_paged_tiles_both(const PagedArgs& p, hipStream_t stream) { return launch_tiles<uint16_t, kCap | kBias>(p, stream); }

}  // namespace attnw
