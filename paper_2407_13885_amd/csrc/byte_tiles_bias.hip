// Attention over a paged cache in 8 bits by blocks of 128 rows (paged_tiles.h): scores with a bias by distance.
#include "paged_tiles.h"

namespace attnw {

hipError_t launch_byte_tiles_bias(const PagedArgs& p, const ScalesView& scales, hipStream_t stream) { return launch_byte_tiles<uint16_t, kBias>(p, scales, stream); }

}  // namespace attnw
