// The tiled matrix product for f16 operands (la2_linear_tiles.h).
#include "la2_linear_tiles.h"

namespace la2 {
hipError_t launch_product_f16(int tile, bool across_a, bool across_b, const ProductParams& p, hipStream_t s) {
  return linear::launch_product<_Float16>(tile, across_a, across_b, p, s);
}
}  // namespace la2
