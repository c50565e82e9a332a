// Linear layers: z = x w^T + b, y = act(z) + residual, and the gradients
//
//   dz = dy act'(z),  dx = dz w,  dw = dz^T x,  db = sum_rows dz
//
// Many rows: the tiled product (la2_linear_tiles.h), forward with its epilogue, backward twice.  A product whose tiles do not fill the
// device is cut along the reduction; the pieces' fp32 sums meet in the workspace and are joined in a fixed order by a
// launch of its own.  The backward pass forms dz (rounded to the operands' type, as the matrix instructions take it) and the bias'
// gradient (from the unrounded values, fp32) in one pass over dy and z.
//
// Few rows (a decode step's): bound by the bytes of w, each read once, straight into registers (linear_few_kernel).
//
// The tiled product loads 16-byte chunks: an operand whose rows do not start at, or are no, whole chunks is copied to rows that are,
// zeros behind the end, before the product runs (two more passes over that operand, small against the product).
#include <algorithm>

#include "la2_bf16_common.h"
#include "la2_linear.h"

namespace la2 {
namespace {

using bf16k::f32x4;

// ---- few rows
constexpr int kFewRows = 32;
constexpr int kFewWaves = 8;

template <typename E>
__device__ __forceinline__ f32x4 multiply16(typename Piece<E>::vec a, typename Piece<E>::vec b, f32x4 c) {
  return bf16k::mfma16(a, b, c);
}
template <>
__device__ __forceinline__ f32x4 multiply16<float>(Piece<float>::vec a, Piece<float>::vec b, f32x4 c) {
#pragma unroll
  for (int e = 0; e < 4; e++) c = __builtin_amdgcn_mfma_f32_16x16x4f32(a[e], b[e], c, 0, 0, 0);
  return c;
}

// A workgroup forms 16 outputs of IT * 16 rows: its waves share the reduction (a wave's lanes read 4 * 64 bytes of each of 16 rows of w at
// a time), and meet in LDS.  x comes from the caches.
template <typename E, int IT>
__global__ __launch_bounds__(64 * kFewWaves) void linear_few_kernel(ProductParams p) {
  constexpr int N = Piece<E>::N, U = 4;
  __shared__ float part[kFewWaves][IT * 16][16 + 4];
  const int lane = threadIdx.x & 63, w = threadIdx.x >> 6, l16 = lane & 15, g = lane >> 4;
  const int64_t j0 = (int64_t)blockIdx.x * 16;
  const E* wrow = static_cast<const E*>(p.b) + min(j0 + l16, p.J - 1) * p.ldb;
  const int64_t wwidth = j0 + l16 < p.J ? p.R : 0;
  f32x4 acc[IT];
#pragma unroll
  for (int t = 0; t < IT; t++) acc[t] = f32x4{0.f, 0.f, 0.f, 0.f};
  for (int64_t k = (int64_t)w * (4 * U * N); k < p.R; k += kFewWaves * 4 * U * N) {
    typename Piece<E>::vec fw[U], fx[IT][U];
#pragma unroll
    for (int u = 0; u < U; u++) fw[u] = Piece<E>::raw(wrow, k + (4 * u + g) * N, wwidth);
#pragma unroll
    for (int t = 0; t < IT; t++) {
      const int64_t i = 16 * t + l16;
      const E* xrow = static_cast<const E*>(p.a) + min(i, p.I - 1) * p.lda;
#pragma unroll
      for (int u = 0; u < U; u++) fx[t][u] = Piece<E>::raw(xrow, k + (4 * u + g) * N, i < p.I ? p.R : 0);
    }
#pragma unroll
    for (int t = 0; t < IT; t++)
#pragma unroll
      for (int u = 0; u < U; u++) acc[t] = multiply16<E>(fw[u], fx[t][u], acc[t]);
  }
#pragma unroll
  for (int t = 0; t < IT; t++) *reinterpret_cast<f32x4*>(&part[w][16 * t + l16][4 * g]) = acc[t];
  __syncthreads();
  constexpr int PIECES = 16 / N;
  if ((int)threadIdx.x < IT * 16 * PIECES) {
    const int i = threadIdx.x / PIECES, c = threadIdx.x % PIECES * N;
    if (i < p.I && j0 + c < p.J) {
      float v[N];
#pragma unroll
      for (int e = 0; e < N; e++) {
        v[e] = 0.f;
#pragma unroll
        for (int k = 0; k < kFewWaves; k++) v[e] += part[k][i][c + e];
      }
      finish<E, N>(p, i, j0 + c, v);
    }
  }
}

// ---- the pieces of a cut reduction
template <typename E>
__global__ __launch_bounds__(256) void linear_join_kernel(ProductParams p) {
  constexpr int N = Piece<E>::N;
  const int64_t pieces = (p.J + N - 1) / N, at = (int64_t)blockIdx.x * 256 + threadIdx.x;
  if (at >= p.I * pieces) return;
  const int64_t i = at / pieces, j = at % pieces * N;
  const int left = (int)min(p.J - j, (int64_t)N);
  float v[N];
#pragma unroll
  for (int e = 0; e < N; e++) v[e] = 0.f;
  for (int s = 0; s < p.splits; s++) {
    const float* from = p.partial + (s * p.I + i) * p.J + j;
#pragma unroll
    for (int e = 0; e < N; e++)
      if (e < left) v[e] += from[e];
  }
  finish<E, N>(p, i, j, v);
}

// ---- operands with rows of whole chunks
template <typename E>
__global__ __launch_bounds__(256) void linear_pad_kernel(const E* from, int64_t ld, int64_t rows, int32_t width, E* to, int64_t ldo) {
  constexpr int N = Piece<E>::N;
  const int64_t pieces = ldo / N, at = (int64_t)blockIdx.x * 256 + threadIdx.x;
  if (at >= rows * pieces) return;
  const int64_t row = at / pieces, col = at % pieces * N;
  *reinterpret_cast<typename Piece<E>::vec*>(to + row * ldo + col) = Piece<E>::raw(from + row * ld, col, width);
}

// ---- dz and the bias' gradient
constexpr int kSlopeCols = 32, kSlopeRows = 8;   // lanes along a row (a piece each), rows at a time
struct SlopeParams {
  int64_t rows;
  int32_t width, act;
  int64_t ld, ldo;
  const void *dy, *pre;
  void* dz;         // nullptr: sums only
  float* partial;   // [gridDim.y][width], nullptr: dz only
};
template <typename E>
__global__ __launch_bounds__(kSlopeCols * kSlopeRows) void linear_slope_kernel(SlopeParams p) {
  constexpr int N = Piece<E>::N;
  __shared__ float part[kSlopeRows][kSlopeCols * N + 1];
  const int lane = threadIdx.x % kSlopeCols, sub = threadIdx.x / kSlopeCols;
  const int col = (blockIdx.x * kSlopeCols + lane) * N;
  float sum[N];
#pragma unroll
  for (int e = 0; e < N; e++) sum[e] = 0.f;
  if (col < p.width) {
    for (int64_t row = (int64_t)blockIdx.y * kSlopeRows + sub; row < p.rows; row += (int64_t)gridDim.y * kSlopeRows) {
      float g[N];
      Piece<E>::load(static_cast<const E*>(p.dy) + row * p.ld, col, p.width, g);
      if (p.act != kActNone) {
        float z[N];
        Piece<E>::load(static_cast<const E*>(p.pre) + row * p.ld, col, p.width, z);
#pragma unroll
        for (int e = 0; e < N; e++) g[e] *= col + e < p.width ? act_slope(z[e], p.act) : 0.f;
      }
#pragma unroll
      for (int e = 0; e < N; e++) sum[e] += g[e];
      if (p.dz != nullptr) Piece<E>::store(static_cast<E*>(p.dz) + row * p.ldo, col, (int)p.ldo, g);   // zeros up to ldo
    }
  }
  if (p.partial == nullptr) return;
#pragma unroll
  for (int e = 0; e < N; e++) part[sub][lane * N + e] = sum[e];
  __syncthreads();
  for (int c = threadIdx.x; c < kSlopeCols * N; c += kSlopeCols * kSlopeRows) {
    const int j = blockIdx.x * kSlopeCols * N + c;
    if (j >= p.width) continue;
    float s = 0.f;
#pragma unroll
    for (int r = 0; r < kSlopeRows; r++) s += part[r][c];
    p.partial[(int64_t)blockIdx.y * p.width + j] = s;
  }
}

// ---- host side
size_t elem(int dtype) { return dtype == kF32 ? 4 : 2; }
int64_t up(int64_t x, int64_t to) { return (x + to - 1) / to * to; }
int64_t chunk(int dtype) { return dtype == kF32 ? 4 : 8; }   // elements of 16 bytes
bool whole_chunks(int dtype, int64_t ld, int64_t width) { return width == 0 || (ld % chunk(dtype) == 0 && width % chunk(dtype) == 0); }

// Takes pieces of the workspace, each from a multiple of 256 bytes on; without a workspace it only counts.
struct Taker {
  char* base;
  size_t used = 0;
  void* take(size_t bytes) {
    void* at = base == nullptr ? nullptr : base + used;
    used += (bytes + 255) / 256 * 256;
    return at;
  }
};

struct Plan {
  int tile;
  int32_t splits;
  int64_t span;
};
// The tile and the number of pieces of the reduction with the least time by this estimate: a unit works off its workgroups at a rate
// that grows with the tile, a workgroup has a start and an end, and the pieces' sums are written and read once more.
Plan plan_product(int dtype, int64_t I, int64_t J, int64_t R, int units) {
  const int step = dtype == kF32 ? 32 : 64;
  const int64_t steps = std::max<int64_t>(1, (R + step - 1) / step);
  Plan best{kTile64, 1, up(std::max<int64_t>(R, 1), step)};
  double least = 1e30;
  for (int tile = kTile64; tile <= kTile256; tile++) {
    const int64_t T = 64 << tile;
    const double per_step = (dtype == kF32 ? 30.0 : 2.1) * (double)(T * T) / 65536.0 / (tile == kTile256 ? 1.0 : tile == kTile128 ? 0.8 : 0.4);
    const int64_t tiles = ((I + T - 1) / T) * ((J + T - 1) / T);
    if (tiles > 0x3FFFFFFF) continue;
    for (int64_t splits = 1; splits <= 32 && splits <= steps; splits *= 2) {
      const int64_t span = (steps + splits - 1) / splits, n = (steps + span - 1) / span;
      if (n != splits && n < splits) continue;
      const int64_t rounds = (tiles * n + units - 1) / units;
      double t = rounds * (span * per_step + 1.0) + 2.0;
      if (n > 1) t += 4.0 + (double)I * (double)J * 4.0 * (2.0 * n) / 4e6;
      if (n > 1 && (double)I * J * n * 4.0 > 512e6) continue;
      if (t < least) {
        least = t;
        best = Plan{tile, (int32_t)n, span * step};
      }
    }
  }
  return best;
}

template <typename E>
hipError_t join(const ProductParams& p, hipStream_t s) {
  const int64_t pieces = p.I * ((p.J + Piece<E>::N - 1) / Piece<E>::N);
  hipLaunchKernelGGL(linear_join_kernel<E>, dim3((unsigned)((pieces + 255) / 256)), dim3(256), 0, s, p);
  return hipGetLastError();
}

// One product; the operands are of whole chunks.  `t`: where the pieces' sums are taken from.
hipError_t product(int dtype, bool across_a, bool across_b, ProductParams p, Taker& t, bool count_only, int units, hipStream_t s) {
  if (p.I == 0 || p.J == 0) return hipSuccess;
  const Plan plan = plan_product(dtype, p.I, p.J, p.R, units);
  p.splits = plan.splits;
  p.span = plan.span;
  p.partial = plan.splits > 1 ? static_cast<float*>(t.take((size_t)p.I * p.J * plan.splits * 4)) : nullptr;
  if (count_only) return hipSuccess;
  hipError_t e = dtype == kBF16  ? launch_product_bf16(plan.tile, across_a, across_b, p, s)
                 : dtype == kF16 ? launch_product_f16(plan.tile, across_a, across_b, p, s)
                                 : launch_product_f32(plan.tile, across_a, across_b, p, s);
  if (e != hipSuccess || plan.splits == 1) return e;
  return dtype == kBF16 ? join<__bf16>(p, s) : dtype == kF16 ? join<_Float16>(p, s) : join<float>(p, s);
}

template <typename E>
void pad_rows(const void* from, int64_t ld, int64_t rows, int64_t width, void* to, int64_t ldo, hipStream_t s) {
  const int64_t pieces = rows * (ldo / Piece<E>::N);
  hipLaunchKernelGGL(linear_pad_kernel<E>, dim3((unsigned)((pieces + 255) / 256)), dim3(256), 0, s, static_cast<const E*>(from), ld, rows,
                     (int32_t)width, static_cast<E*>(to), ldo);
}

// An operand in whole chunks: itself, or a copy in the workspace.
hipError_t regular(int dtype, const void*& at, int64_t& ld, int64_t rows, int64_t width, Taker& t, bool count_only, hipStream_t s) {
  if (whole_chunks(dtype, ld, width)) return hipSuccess;
  const int64_t ldo = up(width, chunk(dtype));
  void* to = t.take((size_t)rows * ldo * elem(dtype));
  if (!count_only && rows > 0) {
    if (dtype == kF32) pad_rows<float>(at, ld, rows, width, to, ldo, s);
    else pad_rows<__bf16>(at, ld, rows, width, to, ldo, s);   // copies bits: either 16-bit type
  }
  at = to;
  ld = ldo;
  return count_only ? hipSuccess : hipGetLastError();
}

template <typename E>
hipError_t few(const ProductParams& p, hipStream_t s) {
  const dim3 grid((unsigned)((p.J + 15) / 16)), block(64 * kFewWaves);
  if (p.I <= 16) hipLaunchKernelGGL((linear_few_kernel<E, 1>), grid, block, 0, s, p);
  else hipLaunchKernelGGL((linear_few_kernel<E, 2>), grid, block, 0, s, p);
  return hipGetLastError();
}

hipError_t forward(const LinearParams& q, Taker& t, bool count_only, int units, hipStream_t s) {
  ProductParams p{};
  p.I = q.rows;
  p.J = q.out;
  p.R = q.in;
  p.a = q.x;
  p.b = q.w;
  p.lda = q.stride_x;
  p.ldb = q.stride_w;
  p.bias = q.bias;
  p.residual = q.residual;
  p.out = q.y;
  p.pre = q.pre;
  p.ldo = q.stride_y;
  p.act = q.act;
  p.splits = 1;
  if (q.rows <= kFewRows) {
    if (count_only) return hipSuccess;
    return q.dtype == kBF16 ? few<__bf16>(p, s) : q.dtype == kF16 ? few<_Float16>(p, s) : few<float>(p, s);
  }
  hipError_t e = regular(q.dtype, p.a, p.lda, q.rows, q.in, t, count_only, s);
  if (e == hipSuccess) e = regular(q.dtype, p.b, p.ldb, q.out, q.in, t, count_only, s);
  if (e == hipSuccess) e = product(q.dtype, false, false, p, t, count_only, units, s);
  return e;
}

template <typename E>
void slope(const SlopeParams& p, dim3 grid, hipStream_t s) {
  hipLaunchKernelGGL(linear_slope_kernel<E>, grid, dim3(kSlopeCols * kSlopeRows), 0, s, p);
}

hipError_t backward(const LinearParams& q, Taker& t, bool count_only, int units, hipStream_t s) {
  const int d = q.dtype;
  const bool products = q.dx != nullptr || q.dw != nullptr;
  const void* dz = q.dy;
  int64_t ldz = q.stride_y;
  SlopeParams sp{};
  sp.rows = q.rows;
  sp.width = q.out;
  sp.act = q.act;
  sp.ld = q.stride_y;
  sp.dy = q.dy;
  sp.pre = q.pre;
  const bool own = products && (q.act != kActNone || !whole_chunks(d, q.stride_y, q.out));
  if (own) {
    ldz = up(q.out, chunk(d));
    dz = sp.dz = t.take((size_t)q.rows * ldz * elem(d));
  }
  sp.ldo = ldz;
  if (q.out > 0 && (own || q.d_bias != nullptr)) {
    const int64_t cols = (q.out + kSlopeCols * chunk(d) - 1) / (kSlopeCols * chunk(d));
    const int64_t blocks = std::max<int64_t>(1, std::min<int64_t>((q.rows + kSlopeRows - 1) / kSlopeRows, (int64_t)units * 8 / cols));
    if (q.d_bias != nullptr) sp.partial = static_cast<float*>(t.take((size_t)blocks * q.out * 4));
    if (!count_only) {
      const dim3 grid((unsigned)cols, (unsigned)blocks);
      if (d == kBF16) slope<__bf16>(sp, grid, s);
      else if (d == kF16) slope<_Float16>(sp, grid, s);
      else slope<float>(sp, grid, s);
      hipError_t e = hipGetLastError();
      if (e == hipSuccess && q.d_bias != nullptr) e = launch_column_sums(sp.partial, blocks, q.out, q.out, q.d_bias, nullptr, s);
      if (e != hipSuccess) return e;
    }
  }
  if (q.dx != nullptr) {
    ProductParams p{};
    p.I = q.rows;
    p.J = q.in;
    p.R = q.out;
    p.a = dz;
    p.lda = ldz;
    p.b = q.w;
    p.ldb = q.stride_w;
    p.out = q.dx;
    p.ldo = q.stride_x;
    hipError_t e = regular(d, p.b, p.ldb, q.out, q.in, t, count_only, s);
    if (e == hipSuccess) e = product(d, false, true, p, t, count_only, units, s);
    if (e != hipSuccess) return e;
  }
  if (q.dw != nullptr) {
    ProductParams p{};
    p.I = q.out;
    p.J = q.in;
    p.R = q.rows;
    p.a = dz;
    p.lda = ldz;
    p.b = q.x;
    p.ldb = q.stride_x;
    p.out = q.dw;
    p.ldo = q.stride_w;
    hipError_t e = regular(d, p.b, p.ldb, q.rows, q.in, t, count_only, s);
    if (e == hipSuccess) e = product(d, true, true, p, t, count_only, units, s);
    if (e != hipSuccess) return e;
  }
  return hipSuccess;
}

}  // namespace

size_t linear_fwd_workspace(const LinearParams& p, int units) {
  Taker t{nullptr};
  (void)forward(p, t, true, units, nullptr);
  return t.used;
}
size_t linear_bwd_workspace(const LinearParams& p, int units) {
  Taker t{nullptr};
  (void)backward(p, t, true, units, nullptr);
  return t.used;
}
hipError_t launch_linear_fwd(const LinearParams& p, void* workspace, int units, hipStream_t s) {
  Taker t{static_cast<char*>(workspace)};
  return forward(p, t, false, units, s);
}
hipError_t launch_linear_bwd(const LinearParams& p, void* workspace, int units, hipStream_t s) {
  Taker t{static_cast<char*>(workspace)};
  return backward(p, t, false, units, s);
}

}  // namespace la2
