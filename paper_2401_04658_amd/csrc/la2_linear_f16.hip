// The tiled matrix products of f16 operands (la2_linear_tiles.h).
#include "la2_linear_tiles.h"

namespace la2 {
hipError_t launch_product_f16(int tile, const ProductParams& p, hipStream_t s) { return linear::launch_product<_Float16>(tile, p, s); }
hipError_t launch_pair_f16(int tile, const PairParams& p, hipStream_t s) { return linear::launch_pair<_Float16>(tile, p, s); }
}  // namespace la2
