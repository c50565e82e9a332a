// Linear layers: z = x w^T + b, y = act(z) + residual, and the gradients
//
//   dz = dy act'(z),  dx = dz w,  dw = dz^T x,  db = sum_rows dz
//
// Many rows: the tiled product (la2_linear_tiles.h), forward with its epilogue, backward both in one launch.  A product whose tiles do not fill the
// device is cut along the reduction; the pieces' fp32 sums meet in the workspace and are joined in a fixed order by a
// launch of its own.  The backward pass forms dz (rounded to the operands' type, as the matrix instructions take it) and the bias'
// gradient (from the unrounded values, fp32) in one pass over dy and z.
//
// Few rows (a decode step's): bound by the bytes of w, each read once, straight into registers (linear_few_kernel).
//
// The tiled product loads 16-byte chunks: an operand whose rows do not start at, or are no, whole chunks is copied to rows that are,
// zeros behind the end, before the product runs (two more passes over that operand, small against the product).
#include <algorithm>
#include <cmath>

#include "la2_bf16_common.h"
#include "la2_linear.h"

namespace la2 {
namespace {

using bf16k::f32x4;

// ---- few rows
constexpr int kFewRows = 32;
constexpr int kFewWaves = 8;
// Up to 16 rows, unless few outputs leave units without work for a long reduction (16 rows, 8192 features into 2048, bf16: 16.8 us, the tiled
// product with a cut reduction 12.0); up to 32 where the weight is small (32 x 2048 x 2048 7.8 against 8.6, 32 x 8192 x 8192 48 against 34).
bool few_rows(int64_t rows, int64_t in, int64_t out, int units) {
  if (rows <= 16) return out >= 16 * (int64_t)units || in <= 4096;
  return rows <= kFewRows && in * out <= (int64_t)1 << 22;
}

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
  // A wave works off a stretch of its own, and each workgroup starts its stretches at another place: rows that are a power of two apart
  // would all be read from the same memory channels at a time (8192 x 8192 bf16, one row of x: 38 us in step, 30 so)
  constexpr int64_t UNIT = 4 * U * N;
  const int turns = (int)(((p.R + UNIT - 1) / UNIT + kFewWaves - 1) / kFewWaves);
  int turn = turns > 0 ? (int)(blockIdx.x % (unsigned)turns) : 0;
  for (int n = 0; n < turns; n++, turn = turn + 1 == turns ? 0 : turn + 1) {
    const int64_t k = (int64_t)(w * turns + turn) * UNIT;
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
      float b[N];
      load_floats(p.bias, j0 + c, p.J, 0.f, b);
      with_act(p.act, [&](auto act) { finish<E, decltype(act)::value, N>(p, i, j0 + c, b, v); });
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
  float v[N], b[N];
#pragma unroll
  for (int e = 0; e < N; e++) v[e] = 0.f;
#pragma unroll 4
  for (int s = 0; s < p.splits; s++) {
    float from[N];
    load_any_floats(p.partial + (s * p.I + i) * p.J, j, p.J, from);
#pragma unroll
    for (int e = 0; e < N; e++) v[e] += from[e];
  }
  load_floats(p.bias, j, p.J, 0.f, b);
  with_act(p.act, [&](auto act) { finish<E, decltype(act)::value, N>(p, i, j, b, v); });
}

// ---- in front of the products: dz and the rows' shares of the bias' gradient, operands copied to rows of whole chunks
constexpr int kSlopeCols = 32, kSlopeRows = 8;   // lanes along a row (a piece each), rows at a time
struct PadParams {
  const void* from;
  void* to;
  int64_t ld, ldo, rows;
  int32_t width, groups;   // workgroups; 0: nothing to copy
};
struct PrepareParams {
  int64_t rows;            // of dz
  int32_t width, act;
  int64_t ld, ldo;
  const void *dy, *pre;
  void* dz;                // nullptr: sums only
  float* partial;          // [slope_rows][width], nullptr: dz only
  int32_t slope_cols, slope_rows;   // workgroups along a row and along the rows; 0: neither
  PadParams pad[2];
};
template <typename E>
__device__ __forceinline__ void pad_rows(const PadParams& p, uint32_t wg) {
  constexpr int N = Piece<E>::N;
  const int64_t pieces = p.ldo / N;
  for (int64_t at = (int64_t)wg * 256 + threadIdx.x; at < p.rows * pieces; at += (int64_t)p.groups * 256) {
    const int64_t row = at / pieces, col = at % pieces * N;
    *reinterpret_cast<typename Piece<E>::vec*>(static_cast<E*>(p.to) + row * p.ldo + col) =
        Piece<E>::raw(static_cast<const E*>(p.from) + row * p.ld, col, p.width);
  }
}
template <typename E>
__global__ __launch_bounds__(kSlopeCols * kSlopeRows) void linear_prepare_kernel(PrepareParams p) {
  constexpr int N = Piece<E>::N;
  __shared__ float part[kSlopeRows][kSlopeCols * N + 1];
  uint32_t wg = blockIdx.x;
  const uint32_t slopes = (uint32_t)p.slope_cols * (uint32_t)p.slope_rows;
  if (wg >= slopes) {
    wg -= slopes;
    if (wg < (uint32_t)p.pad[0].groups) pad_rows<E>(p.pad[0], wg);
    else pad_rows<E>(p.pad[1], wg - (uint32_t)p.pad[0].groups);
    return;
  }
  const int lane = threadIdx.x % kSlopeCols, sub = threadIdx.x / kSlopeCols;
  const int strip = (int)(wg % (uint32_t)p.slope_cols), share = (int)(wg / (uint32_t)p.slope_cols);
  const int col = (strip * kSlopeCols + lane) * N;
  float sum[N];
#pragma unroll
  for (int e = 0; e < N; e++) sum[e] = 0.f;
  if (col < p.width) {
    with_act(p.act, [&](auto act) {
      constexpr int ACT = decltype(act)::value;
#pragma unroll 2
      for (int64_t row = (int64_t)share * kSlopeRows + sub; row < p.rows; row += (int64_t)p.slope_rows * kSlopeRows) {
        float g[N];
        Piece<E>::load(static_cast<const E*>(p.dy) + row * p.ld, col, p.width, g);
        if (ACT != kActNone) {   // (behind the row's end g is 0 and the slope that of 0)
          float z[N];
          Piece<E>::load(static_cast<const E*>(p.pre) + row * p.ld, col, p.width, z);
#pragma unroll
          for (int e = 0; e < N; e++) g[e] *= act_slope<ACT>(z[e]);
        }
#pragma unroll
        for (int e = 0; e < N; e++) sum[e] += g[e];
        if (p.dz != nullptr) Piece<E>::store(static_cast<E*>(p.dz) + row * p.ldo, col, (int)p.ldo, g);   // zeros up to ldo
      }
    });
  }
  if (p.partial == nullptr) return;
#pragma unroll
  for (int e = 0; e < N; e++) part[sub][lane * N + e] = sum[e];
  __syncthreads();
  for (int c = threadIdx.x; c < kSlopeCols * N; c += kSlopeCols * kSlopeRows) {
    const int j = strip * kSlopeCols * N + c;
    if (j >= p.width) continue;
    float s = 0.f;
#pragma unroll
    for (int r = 0; r < kSlopeRows; r++) s += part[r][c];
    p.partial[(int64_t)share * p.width + j] = s;
  }
}

// ---- host side
size_t elem(int dtype) { return dtype == kF32 ? 4 : 2; }
int64_t up(int64_t x, int64_t to) { return (x + to - 1) / to * to; }
int64_t chunk(int dtype) { return dtype == kF32 ? 4 : 8; }   // elements of 16 bytes
bool whole_chunks(int dtype, int64_t ld, int64_t width) { return width == 0 || (ld % chunk(dtype) == 0 && width % chunk(dtype) == 0); }

// Outputs that do not fit the memory-side cache (256 MiB) are stored past the caches: 16384 x 8192 bf16 with its sums kept 547 us against 561.
bool past_caches(int64_t rows, int64_t width, int dtype) { return rows * width * (int64_t)elem(dtype) >= (int64_t)256 << 20; }

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

// ---- how a product is cut
struct Plan {
  int tile = kTile64;
  int32_t splits[2] = {1, 1};
  int64_t span[2] = {0, 0};
};
struct Extent {
  int64_t I, J, R;
};
// Microseconds of a workgroup with a unit for itself per reduction step, of a unit with several of them per workgroup and step, and of
// a workgroup's start and end.  Measured on 64 to 8192 rows of 2048 features into 2048 (bf16; fp32, whose steps are half as long).
struct TileCost {
  double alone, shared, ends;
};
constexpr TileCost kCost16[kTiles] = {{0.29, 0.21, 0.9}, {0.60, 0.52, 2.0}, {1.45, 1.75, 8.0}};
constexpr TileCost kCost32[kTiles] = {{0.63, 0.56, 1.0}, {2.0, 1.98, 2.0}, {7.4, 7.4, 6.0}};

// The tile, and for each of the `count` products of a launch the number of pieces of its reduction, with the least time by these costs.  Pieces
// are as long as a unit's share of all steps, or twice that, or whole; their sums are written and read once more (about 12 bytes
// a nanosecond, they stay in the caches) and joined by a launch of its own.
Plan plan_products(int dtype, const Extent* e, int count, int units) {
  const int step = dtype == kF32 ? 32 : 64;
  Plan best;
  double least = 1e30;
  for (int tile = kTile64; tile < kTiles; tile++) {
    const TileCost& cost = (dtype == kF32 ? kCost32 : kCost16)[tile];
    const int64_t T = 64 << tile;
    int64_t steps[2], tiles[2], all = 0;
    for (int k = 0; k < count; k++) {
      steps[k] = std::max<int64_t>(1, (e[k].R + step - 1) / step);
      tiles[k] = ((e[k].I + T - 1) / T) * ((e[k].J + T - 1) / T);
      all += steps[k] * tiles[k];
    }
    for (int cut = 0; cut < 3; cut++) {
      const int64_t most = cut == 0 ? INT64_MAX : std::max<int64_t>(4, (all + units - 1) / units) * cut;
      Plan plan;
      plan.tile = tile;
      double work = 0, longest = 0, shortest = 1e30, sums = 0, time = 3.0;
      int64_t groups = 0;
      bool cuts = false;
      for (int k = 0; k < count; k++) {
        const int64_t want = std::min<int64_t>(32, steps[k] <= most ? 1 : (steps[k] + most - 1) / most);
        const int64_t span = (steps[k] + want - 1) / want, n = (steps[k] + span - 1) / span;
        plan.span[k] = span * step;
        plan.splits[k] = (int32_t)n;
        const double one = span * cost.shared + cost.ends;
        work += (double)(tiles[k] * n) * one;
        longest = std::max(longest, std::max(one, span * cost.alone + cost.ends));
        shortest = std::min(shortest, one);
        groups += tiles[k] * n;
        if (n > 1) {
          cuts = true;
          sums += (double)e[k].I * (double)e[k].J * n * 4.0;
          time += 4.5;
        }
      }
      if (cut > 0 && (!cuts || sums > 512e6)) continue;
      if ((groups + kMostSumGroups) * kTileThreads[tile] > kMostThreads) continue;   // (the 256 tile, not cut, always stays: linear_fits)
      const double share = work / units;
      if (groups <= units) time += longest;
      else if (count == 1) time += std::max(longest, std::ceil((double)groups / units) * shortest);
      else time += std::max(longest, share + 0.5 * shortest);
      time += 2.0 * sums / 12e6;
      if (time < least) {
        least = time;
        best = plan;
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
hipError_t join_of(int dtype, const ProductParams& p, hipStream_t s) {
  return dtype == kBF16 ? join<__bf16>(p, s) : dtype == kF16 ? join<_Float16>(p, s) : join<float>(p, s);
}

// The plan's part of product k, and where its pieces' sums go
void apply(const Plan& plan, int k, ProductParams& p, Taker& t) {
  p.splits = plan.splits[k];
  p.span = plan.span[k];
  p.partial = p.splits > 1 ? static_cast<float*>(t.take((size_t)p.I * p.J * p.splits * 4)) : nullptr;
}

// An operand in whole chunks: itself, or a copy in the workspace that `pad` makes.
void regular(int dtype, const void*& at, int64_t& ld, int64_t rows, int64_t width, Taker& t, PadParams& pad) {
  if (whole_chunks(dtype, ld, width)) return;
  const int64_t ldo = up(width, chunk(dtype)), pieces = rows * (ldo / chunk(dtype));
  pad.from = at;
  pad.to = t.take((size_t)rows * ldo * elem(dtype));
  pad.ld = ld;
  pad.ldo = ldo;
  pad.rows = rows;
  pad.width = (int32_t)width;
  pad.groups = (int32_t)std::min<int64_t>((pieces + 255) / 256, 1 << 20);
  at = pad.to;
  ld = ldo;
}

hipError_t prepare(int dtype, const PrepareParams& p, hipStream_t s) {
  const int64_t groups = (int64_t)p.slope_cols * p.slope_rows + p.pad[0].groups + p.pad[1].groups;
  if (groups == 0) return hipSuccess;
  const dim3 grid((unsigned)groups), block(kSlopeCols * kSlopeRows);
  if (dtype == kF32) hipLaunchKernelGGL(linear_prepare_kernel<float>, grid, block, 0, s, p);
  else if (dtype == kBF16) hipLaunchKernelGGL(linear_prepare_kernel<__bf16>, grid, block, 0, s, p);
  else hipLaunchKernelGGL(linear_prepare_kernel<_Float16>, grid, block, 0, s, p);
  return hipGetLastError();
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
  p.past = past_caches(q.rows, q.out, q.dtype);
  p.splits = 1;
  if (p.I == 0 || p.J == 0) return hipSuccess;
  if (few_rows(q.rows, q.in, q.out, units)) {
    if (count_only) return hipSuccess;
    return q.dtype == kBF16 ? few<__bf16>(p, s) : q.dtype == kF16 ? few<_Float16>(p, s) : few<float>(p, s);
  }
  PrepareParams pre{};
  regular(q.dtype, p.a, p.lda, q.rows, q.in, t, pre.pad[0]);
  regular(q.dtype, p.b, p.ldb, q.out, q.in, t, pre.pad[1]);
  const Extent e{p.I, p.J, p.R};
  const Plan plan = plan_products(q.dtype, &e, 1, units);
  apply(plan, 0, p, t);
  if (count_only) return hipSuccess;
  hipError_t st = prepare(q.dtype, pre, s);
  if (st != hipSuccess) return st;
  st = q.dtype == kBF16  ? launch_product_bf16(plan.tile, p, s)
       : q.dtype == kF16 ? launch_product_f16(plan.tile, p, s)
                         : launch_product_f32(plan.tile, p, s);
  return st != hipSuccess || p.splits == 1 ? st : join_of(q.dtype, p, s);
}

hipError_t backward(const LinearParams& q, Taker& t, bool count_only, int units, hipStream_t s) {
  const int d = q.dtype;
  const bool dx = q.dx != nullptr && q.rows > 0 && q.in > 0, dw = q.dw != nullptr && q.out > 0 && q.in > 0;
  const bool db = q.d_bias != nullptr && q.out > 0;
  const void* dz = q.dy;
  int64_t ldz = q.stride_y;
  PrepareParams pre{};
  pre.rows = q.rows;
  pre.width = q.out;
  pre.act = q.act;
  pre.ld = q.stride_y;
  pre.dy = q.dy;
  pre.pre = q.pre;
  const bool own = (dx || dw) && q.out > 0 && q.rows > 0 && (q.act != kActNone || !whole_chunks(d, q.stride_y, q.out));
  if (own) {
    ldz = up(q.out, chunk(d));
    dz = pre.dz = t.take((size_t)q.rows * ldz * elem(d));
  }
  pre.ldo = ldz;
  if (own || db) {
    const int64_t strip = kSlopeCols * chunk(d);
    pre.slope_cols = (int32_t)((q.out + strip - 1) / strip);
    pre.slope_rows = (int32_t)std::max<int64_t>(1, std::min<int64_t>((q.rows + kSlopeRows - 1) / kSlopeRows, (int64_t)units * 8 / pre.slope_cols));
    if (db) pre.partial = static_cast<float*>(t.take((size_t)pre.slope_rows * q.out * 4));
  }
  PairParams pair{};
  Extent e[2];
  int which[2], count = 0;
  if (dx) {
    ProductParams& p = pair.p[0];
    p.I = q.rows;
    p.J = q.in;
    p.R = q.out;
    p.a = dz;
    p.lda = ldz;
    p.b = q.w;
    p.ldb = q.stride_w;
    p.out = q.dx;
    p.past = past_caches(q.rows, q.in, d);
    p.ldo = q.stride_x;
    regular(d, p.b, p.ldb, q.out, q.in, t, pre.pad[0]);
    e[count] = Extent{p.I, p.J, p.R};
    which[count++] = 0;
  }
  if (dw) {
    ProductParams& p = pair.p[1];
    p.I = q.out;
    p.J = q.in;
    p.R = q.rows;
    p.a = dz;
    p.lda = ldz;
    p.b = q.x;
    p.ldb = q.stride_x;
    p.out = q.dw;
    p.past = past_caches(q.out, q.in, d);
    p.ldo = q.stride_w;
    regular(d, p.b, p.ldb, q.rows, q.in, t, pre.pad[1]);
    e[count] = Extent{p.I, p.J, p.R};
    which[count++] = 1;
  }
  Plan plan;
  if (count > 0) {
    plan = plan_products(d, e, count, units);
    for (int k = 0; k < count; k++) {
      apply(plan, k, pair.p[which[k]], t);
      pair.groups[which[k]] = 1;
    }
  }
  if (count_only) return hipSuccess;
  hipError_t st = prepare(d, pre, s);
  if (st != hipSuccess) return st;
  if (count == 0) return db ? launch_column_sums(pre.partial, pre.slope_rows, q.out, q.out, q.d_bias, nullptr, s) : hipSuccess;
  if (db) {
    pair.partial = pre.partial;
    pair.count = pre.slope_rows;
    pair.width = q.out;
    pair.sums = q.d_bias;
  }
  st = d == kBF16 ? launch_pair_bf16(plan.tile, pair, s) : d == kF16 ? launch_pair_f16(plan.tile, pair, s) : launch_pair_f32(plan.tile, pair, s);
  for (int k = 0; k < count && st == hipSuccess; k++)
    if (pair.p[which[k]].splits > 1) st = join_of(d, pair.p[which[k]], s);
  return st;
}

}  // namespace

bool linear_fits(const LinearParams& p) {
  const int64_t T = 64 << kTile256, rows = (p.rows + T - 1) / T, in = (p.in + T - 1) / T, out = (p.out + T - 1) / T;
  const int64_t most = kMostThreads / kTileThreads[kTile256] - kMostSumGroups;
  return rows * out <= most && rows * in + out * in <= most;
}

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
