// The tiled matrix products of bf16 operands (la2_linear_tiles.h).
#include "la2_linear_tiles.h"

namespace la2 {
hipError_t launch_product_bf16(int tile, const ProductParams& p, hipStream_t s) { return linear::launch_product<__bf16>(tile, p, s); }
hipError_t launch_pair_bf16(int tile, const PairParams& p, hipStream_t s) { return linear::launch_pair<__bf16>(tile, p, s); }
}  // namespace la2
