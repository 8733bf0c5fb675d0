// The tiles of products with 8-bit weights: instantiations, gated.
#include "w8_tile.h"

namespace laser {

void launch_w8_tile_gated(const W8Args& a, int v, hipStream_t stream) { go_w8_tile<true>(a, v, stream); }

}  // namespace laser
