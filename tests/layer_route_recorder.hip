// Stand-ins for the launchers of the tiled products that write down what they are asked for instead of launching it: linked with the
// host side of the linear layers they show, without a GPU, how a call is planned.  One line a product.  Calls that launch something else beside
// the products (copies, sums, joins) end where they would.
#include <hip/hip_runtime.h>

#include <cstdio>
#include <cstring>
#include <string>

#include "../paper_2401_04658_amd/csrc/la2_linear.h"

namespace {
std::string lines;
hipError_t note(const char* kind, int dtype, int tile, const la2::ProductParams& p) {
  char line[256];
  snprintf(line, sizeof(line), "%s dtype=%d tile=%d I=%lld J=%lld R=%lld splits=%d span=%lld\n", kind, dtype, tile, (long long)p.I, (long long)p.J,
           (long long)p.R, p.splits, (long long)p.span);
  lines += line;
  return hipSuccess;
}
hipError_t both(int dtype, int tile, const la2::PairParams& q) {
  if (q.groups[0] != 0) (void)note("dx", dtype, tile, q.p[0]);
  if (q.groups[1] != 0) (void)note("dw", dtype, tile, q.p[1]);
  return hipSuccess;
}
}  // namespace

extern "C" int routes_take(char* out, int size) {
  const int n = (int)lines.size();
  if (n < size) memcpy(out, lines.c_str(), (size_t)n + 1);
  lines.clear();
  return n < size ? n : -1;
}

namespace la2 {
int device_units() { return 256; }
hipError_t launch_product_bf16(int tile, const ProductParams& p, hipStream_t) { return note("fwd", kBF16, tile, p); }
hipError_t launch_product_f16(int tile, const ProductParams& p, hipStream_t) { return note("fwd", kF16, tile, p); }
hipError_t launch_product_f32(int tile, const ProductParams& p, hipStream_t) { return note("fwd", kF32, tile, p); }
hipError_t launch_pair_bf16(int tile, const PairParams& p, hipStream_t) { return both(kBF16, tile, p); }
hipError_t launch_pair_f16(int tile, const PairParams& p, hipStream_t) { return both(kF16, tile, p); }
hipError_t launch_pair_f32(int tile, const PairParams& p, hipStream_t) { return both(kF32, tile, p); }
hipError_t launch_column_sums(const float*, int64_t, int64_t, int64_t, float*, float*, hipStream_t) { return hipErrorNotSupported; }
hipError_t launch_layer_norm_fwd(int, const LayerNormParams&, int, hipStream_t) { return hipErrorNotSupported; }
hipError_t launch_layer_norm_bwd(int, const LayerNormParams&, int, hipStream_t) { return hipErrorNotSupported; }
int64_t layer_norm_bwd_partials(int, int64_t, int32_t, int) { return 0; }
int beam_select_chunks(int64_t, int32_t, int32_t, int) { return 1; }
hipError_t launch_beam_select(int, BeamSelectParams, int, hipStream_t) { return hipErrorNotSupported; }
hipError_t launch_beam_reorder(const BeamReorderParams&, int, hipStream_t) { return hipErrorNotSupported; }
}  // namespace la2
