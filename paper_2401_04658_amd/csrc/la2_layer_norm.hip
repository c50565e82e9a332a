// Layer normalisation over the features of a row, forward and backward.
//
//   mean = sum_j x_j / W,  rstd = 1 / sqrt(sum_j (x_j - mean)^2 / W + eps),  h = (x - mean) rstd,  y = h w + b
//   g = dy w,  dx = rstd (g - sum_j g_j / W - h sum_j g_j h_j / W),  dw = sum_rows dy h,  db = sum_rows dy
//
// Bound by memory: a row is read once and stays in registers (CH pieces of 16 bytes per lane, TPR lanes a row), so the variance
// is taken around the mean that was just formed.  A group of lanes walks over rows with w, b and, backward, its columns' share of
// dw and db in registers; sums are fp32.  The shares meet in LDS, then in `partial`, which a second launch sums column by column in
// a fixed order: no atomics, the same bits in every run.
//
// 65536 rows of 2048 bf16 features: forward 98 us (5.5 TB/s), backward 145 us (5.6 TB/s, 5 us of it the second launch); a device copy
// reaches 5.3 TB/s.
#include "la2_layer.h"

namespace la2 {
namespace {

template <int TPR>
struct Shape {
  static constexpr int kThreads = TPR > 256 ? TPR : 256;
  static constexpr int kRows = kThreads / TPR;   // rows that a workgroup works on at a time
};

// Sums of a row over its TPR lanes, in every lane.  `red`: one entry per wave; the caller uses two in turn, so that one barrier per
// sum is enough.
template <int TPR>
__device__ __forceinline__ float2 row_sum(float a, float b, float2* red) {
#pragma unroll
  for (int m = 1; m < (TPR < 64 ? TPR : 64); m <<= 1) {
    a += __shfl_xor(a, m);
    b += __shfl_xor(b, m);
  }
  if constexpr (TPR > 64) {
    if ((threadIdx.x & 63) == 0) red[threadIdx.x >> 6] = make_float2(a, b);
    __syncthreads();
    a = b = 0.f;
#pragma unroll
    for (int w = 0; w < TPR / 64; w++) {
      a += red[w].x;
      b += red[w].y;
    }
  }
  return make_float2(a, b);
}

template <typename T, int TPR, int CH, Edge EDGE>
__global__ __launch_bounds__(Shape<TPR>::kThreads) void layer_norm_fwd_kernel(LayerNormParams p) {
  constexpr int N = Piece<T>::N, RPB = Shape<TPR>::kRows;
  __shared__ float2 red[2][TPR > 64 ? TPR / 64 : 1];
  const int lane = threadIdx.x % TPR, sub = threadIdx.x / TPR;
  float w[CH][N], b[CH][N];
#pragma unroll
  for (int c = 0; c < CH; c++) {
    load_floats<N, EDGE != kRagged>(p.weight, (c * TPR + lane) * N, p.width, 1.f, w[c]);
    load_floats<N, EDGE != kRagged>(p.bias, (c * TPR + lane) * N, p.width, 0.f, b[c]);
  }
  const float width = (float)p.width;   // divided by, so that the mean of equal numbers is that number
  for (int64_t row = (int64_t)blockIdx.x * RPB + sub; row < p.rows; row += (int64_t)gridDim.x * RPB) {
    const T* x = static_cast<const T*>(p.x) + row * p.stride;
    const int end = EDGE == kRagged ? renewed(p.width) : p.width;   // a ragged end's masks are formed for every row: kept, they overflow the scalar registers
    typename Piece<T>::vec raw[CH];
#pragma unroll
    for (int c = 0; c < CH; c++) raw[c] = RowPiece<T, EDGE>((c * TPR + lane) * N, end).fetch(x);
    float v[CH][N], s = 0.f, q = 0.f;
#pragma unroll
    for (int c = 0; c < CH; c++) {
      const auto u = RowPiece<T, EDGE>((c * TPR + lane) * N, end).settle(raw[c]);
#pragma unroll
      for (int i = 0; i < N; i++) {
        v[c][i] = (float)u[i];
        s += v[c][i];
      }
    }
    const float mean = row_sum<TPR>(s, 0.f, red[0]).x / width;
#pragma unroll
    for (int c = 0; c < CH; c++) {
      const int at = (c * TPR + lane) * N;
#pragma unroll
      for (int i = 0; i < N; i++) v[c][i] -= mean;
      if (EDGE == kWhole) {
#pragma unroll
        for (int i = 0; i < N; i++) v[c][i] = at < end ? v[c][i] : 0.f;
      } else if (EDGE == kRagged && at + N > end) {
#pragma unroll
        for (int i = 0; i < N; i++) v[c][i] = at + i < end ? v[c][i] : 0.f;
      }
#pragma unroll
      for (int i = 0; i < N; i++) q = fmaf(v[c][i], v[c][i], q);
    }
    const float rstd = 1.f / sqrtf(row_sum<TPR>(q, 0.f, red[1]).x / width + p.eps);
    T* y = static_cast<T*>(p.y) + row * p.stride;
#pragma unroll
    for (int c = 0; c < CH; c++) {
#pragma unroll
      for (int i = 0; i < N; i++) v[c][i] = fmaf(v[c][i] * rstd, w[c][i], b[c][i]);
      RowPiece<T, EDGE>((c * TPR + lane) * N, end).store(y, v[c]);
    }
    if (lane == 0) {
      p.mean[row] = mean;
      p.rstd[row] = rstd;
    }
  }
}

// TPR lanes, the columns' sums of dw (x) and db (y) of a workgroup's rows: to d_weight / d_bias where it is the only workgroup, else
// to its row of partial
template <typename T, int TPR, int CH, Edge EDGE, bool SUMS>
__global__ __launch_bounds__(Shape<TPR>::kThreads) void layer_norm_bwd_kernel(LayerNormParams p) {
  constexpr int N = Piece<T>::N, RPB = Shape<TPR>::kRows;
  __shared__ float2 red[2][TPR > 64 ? TPR / 64 : 1];
  __shared__ __align__(16) float share[RPB > 1 ? 2 * RPB * TPR * CH * N : 4];   // dw, then db: the rows' groups' sums, in the order of columns
  const int lane = threadIdx.x % TPR, sub = threadIdx.x / TPR;
  constexpr bool AHEAD = CH * N <= 16;   // (registers)
  constexpr bool KEEP = CH * N <= 16;   // the weights stay in registers; else they come from the caches, twice a row
  float w[CH][N], aw[CH][N], ab[CH][N];
#pragma unroll
  for (int c = 0; c < CH; c++) {
    if (KEEP) load_floats<N, EDGE != kRagged>(p.weight, (c * TPR + lane) * N, p.width, 1.f, w[c]);
#pragma unroll
    for (int i = 0; i < N; i++) aw[c][i] = ab[c][i] = 0.f;
  }
  const float width = (float)p.width;
  int turn = 0;
  // The row as it is stored (h and g are formed twice rather than kept), and the next one, on its way meanwhile
  typename Piece<T>::vec rx[CH], rg[CH], nx[CH], ng[CH];
  float mean = 0.f, rstd = 0.f, next_mean = 0.f, next_rstd = 0.f;
  const int64_t step = (int64_t)gridDim.x * RPB;
  auto fetch = [&](int64_t row) {
    if (row >= p.rows) return;
    const int end = EDGE == kRagged ? renewed(p.width) : p.width;
    const T* x = static_cast<const T*>(p.x) + row * p.stride;
    const T* dy = static_cast<const T*>(p.dy) + row * p.stride;
#pragma unroll
    for (int c = 0; c < CH; c++) {
      const RowPiece<T, EDGE> piece((c * TPR + lane) * N, end);
      nx[c] = piece.fetch(x);
      ng[c] = piece.fetch(dy);
    }
    next_mean = p.mean[row];
    next_rstd = p.rstd[row];
  };
  int64_t row = (int64_t)blockIdx.x * RPB + sub;
  fetch(row);
  for (; row < p.rows; row += step, turn ^= 1) {
    const int end = EDGE == kRagged ? renewed(p.width) : p.width;
#pragma unroll
    for (int c = 0; c < CH; c++) {
      const RowPiece<T, EDGE> piece((c * TPR + lane) * N, end);
      rx[c] = piece.settle(nx[c]);
      rg[c] = piece.settle(ng[c]);
    }
    mean = next_mean;
    rstd = next_rstd;
    if (AHEAD) fetch(row + step);
    float sg = 0.f, sh = 0.f;
#pragma unroll
    for (int c = 0; c < CH; c++) {
      if (!KEEP) load_floats<N, EDGE != kRagged>(p.weight, (c * TPR + lane) * N, end, 1.f, w[c]);
#pragma unroll
      for (int i = 0; i < N; i++) {   // behind the row's end dy is 0, and h finite in a row that is
        const float h = ((float)rx[c][i] - mean) * rstd, d = (float)rg[c][i], g = d * w[c][i];
        if (SUMS) {
          aw[c][i] = fmaf(d, h, aw[c][i]);
          ab[c][i] += d;
        }
        sg += g;
        sh = fmaf(g, h, sh);
      }
    }
    const float2 s = row_sum<TPR>(sg, sh, red[turn]);
    const float mg = s.x / width, mh = s.y / width;
    const int last = EDGE == kRagged ? renewed(p.width) : p.width;
    T* dx = static_cast<T*>(p.y) + row * p.stride;
#pragma unroll
    for (int c = 0; c < CH; c++) {
      if (CH > 1) {
        rx[c] = renewed(rx[c]);
        rg[c] = renewed(rg[c]);
      }
      if (!KEEP) load_floats<N, EDGE != kRagged>(p.weight, (c * TPR + lane) * N, last, 1.f, w[c]);
      float v[N];
#pragma unroll
      for (int i = 0; i < N; i++) v[i] = rstd * ((float)rg[c][i] * w[c][i] - mg - ((float)rx[c][i] - mean) * rstd * mh);
      RowPiece<T, EDGE>((c * TPR + lane) * N, last).store(dx, v);
    }
    if (!AHEAD) fetch(row + step);
  }
  if (!SUMS || (p.d_weight == nullptr && p.d_bias == nullptr)) return;
  const bool only = gridDim.x == 1;
  float* ow = only ? p.d_weight : p.partial + (int64_t)blockIdx.x * 2 * p.width;
  float* ob = only ? p.d_bias : p.partial + ((int64_t)blockIdx.x * 2 + 1) * p.width;
  if constexpr (RPB > 1) {
    constexpr int COLS = TPR * CH * N;
#pragma unroll
    for (int c = 0; c < CH; c++)
#pragma unroll
      for (int i = 0; i < N; i += 4) {
        const int at = sub * COLS + (c * TPR + lane) * N + i;
        *reinterpret_cast<float4*>(share + at) = make_float4(aw[c][i], aw[c][i + 1], aw[c][i + 2], aw[c][i + 3]);
        *reinterpret_cast<float4*>(share + RPB * COLS + at) = make_float4(ab[c][i], ab[c][i + 1], ab[c][i + 2], ab[c][i + 3]);
      }
    __syncthreads();
    for (int j = threadIdx.x; j < min(COLS, p.width); j += Shape<TPR>::kThreads) {
      float a = 0.f, b = 0.f;
#pragma unroll
      for (int r = 0; r < RPB; r++) {
        a += share[r * COLS + j];
        b += share[(RPB + r) * COLS + j];
      }
      if (ow != nullptr) ow[j] = a;
      if (ob != nullptr) ob[j] = b;
    }
  } else {
#pragma unroll
    for (int c = 0; c < CH; c++) {
      const int at = (c * TPR + lane) * N;
      if (ow != nullptr) store_floats(ow, at, p.width, aw[c]);
      if (ob != nullptr) store_floats(ob, at, p.width, ab[c]);
    }
  }
}

// Rows that no group of lanes holds in registers: they are read again for every pass over them, from the caches.
constexpr int kWideThreads = 1024;
template <typename T>
__global__ __launch_bounds__(kWideThreads) void layer_norm_wide_fwd_kernel(LayerNormParams p) {
  constexpr int N = Piece<T>::N;
  __shared__ float2 red[2][kWideThreads / 64];
  const float width = (float)p.width;
  for (int64_t row = blockIdx.x; row < p.rows; row += gridDim.x) {
    const T* x = static_cast<const T*>(p.x) + row * p.stride;
    T* y = static_cast<T*>(p.y) + row * p.stride;
    float s = 0.f, q = 0.f, v[N], w[N], b[N];
    for (int j = threadIdx.x * N; j < p.width; j += kWideThreads * N) {
      Piece<T>::load(x, j, p.width, v);
#pragma unroll
      for (int i = 0; i < N; i++) s += v[i];
    }
    const float mean = row_sum<kWideThreads>(s, 0.f, red[0]).x / width;
    for (int j = threadIdx.x * N; j < p.width; j += kWideThreads * N) {
      Piece<T>::load(x, j, p.width, v);
#pragma unroll
      for (int i = 0; i < N; i++) q = j + i < p.width ? fmaf(v[i] - mean, v[i] - mean, q) : q;
    }
    const float rstd = 1.f / sqrtf(row_sum<kWideThreads>(q, 0.f, red[1]).x / width + p.eps);
    for (int j = threadIdx.x * N; j < p.width; j += kWideThreads * N) {
      Piece<T>::load(x, j, p.width, v);
      load_floats(p.weight, j, p.width, 1.f, w);
      load_floats(p.bias, j, p.width, 0.f, b);
#pragma unroll
      for (int i = 0; i < N; i++) v[i] = fmaf((v[i] - mean) * rstd, w[i], b[i]);
      Piece<T>::store(y, j, p.width, v);
    }
    if (threadIdx.x == 0) {
      p.mean[row] = mean;
      p.rstd[row] = rstd;
    }
  }
}

template <typename T>
__global__ __launch_bounds__(kWideThreads) void layer_norm_wide_bwd_kernel(LayerNormParams p) {
  constexpr int N = Piece<T>::N;
  __shared__ float2 red[2][kWideThreads / 64];
  const float width = (float)p.width;
  int turn = 0;
  for (int64_t row = blockIdx.x; row < p.rows; row += gridDim.x, turn ^= 1) {
    const T* x = static_cast<const T*>(p.x) + row * p.stride;
    const T* dy = static_cast<const T*>(p.dy) + row * p.stride;
    T* dx = static_cast<T*>(p.y) + row * p.stride;
    const float mean = p.mean[row], rstd = p.rstd[row];
    float sg = 0.f, sh = 0.f, h[N], g[N], w[N];
    for (int j = threadIdx.x * N; j < p.width; j += kWideThreads * N) {
      Piece<T>::load(x, j, p.width, h);
      Piece<T>::load(dy, j, p.width, g);
      load_floats(p.weight, j, p.width, 1.f, w);
#pragma unroll
      for (int i = 0; i < N; i++) {
        sg += g[i] * w[i];
        sh = fmaf(g[i] * w[i], (h[i] - mean) * rstd, sh);
      }
    }
    const float2 s = row_sum<kWideThreads>(sg, sh, red[turn]);
    for (int j = threadIdx.x * N; j < p.width; j += kWideThreads * N) {
      Piece<T>::load(x, j, p.width, h);
      Piece<T>::load(dy, j, p.width, g);
      load_floats(p.weight, j, p.width, 1.f, w);
#pragma unroll
      for (int i = 0; i < N; i++) g[i] = rstd * (g[i] * w[i] - s.x / width - (h[i] - mean) * rstd * (s.y / width));
      Piece<T>::store(dx, j, p.width, g);
    }
  }
}

// ... and their columns' sums: workgroup (x, y) sums 32 pieces of columns over every gridDim.y-th group of 8 rows
constexpr int kWideCols = 32, kWideRows = 8;
template <typename T>
__global__ __launch_bounds__(kWideCols * kWideRows) void layer_norm_wide_columns_kernel(LayerNormParams p) {
  constexpr int N = Piece<T>::N;
  __shared__ float2 part[kWideRows][kWideCols * N + 1];
  const int lane = threadIdx.x % kWideCols, sub = threadIdx.x / kWideCols, first = blockIdx.x * kWideCols * N, at = first + lane * N;
  float aw[N], ab[N];
#pragma unroll
  for (int i = 0; i < N; i++) aw[i] = ab[i] = 0.f;
  if (at < p.width) {
#pragma unroll 2
    for (int64_t row = (int64_t)blockIdx.y * kWideRows + sub; row < p.rows; row += (int64_t)gridDim.y * kWideRows) {
      const float mean = p.mean[row], rstd = p.rstd[row];
      float h[N], g[N];
      Piece<T>::load(static_cast<const T*>(p.x) + row * p.stride, at, p.width, h);
      Piece<T>::load(static_cast<const T*>(p.dy) + row * p.stride, at, p.width, g);
#pragma unroll
      for (int i = 0; i < N; i++) {
        aw[i] = fmaf(g[i], (h[i] - mean) * rstd, aw[i]);
        ab[i] += g[i];
      }
    }
  }
#pragma unroll
  for (int i = 0; i < N; i++) part[sub][lane * N + i] = make_float2(aw[i], ab[i]);
  __syncthreads();
  for (int c = threadIdx.x; c < kWideCols * N && first + c < p.width; c += kWideCols * kWideRows) {
    float a = 0.f, b = 0.f;
#pragma unroll
    for (int r = 0; r < kWideRows; r++) {
      a += part[r][c].x;
      b += part[r][c].y;
    }
    p.partial[(int64_t)blockIdx.y * 2 * p.width + first + c] = a;
    p.partial[((int64_t)blockIdx.y * 2 + 1) * p.width + first + c] = b;
  }
}

template <int TPR, int CH>
struct Split {
  static constexpr int tpr = TPR, ch = CH;
  // backward: so many elements of a row do not fit the registers beside their columns' sums, which are then formed in a pass of their
  // own and need no scratch memory.  16384 bf16 features: 512 rows 30 us so, 46 with the sums in scratch; 8192 rows 272, 217
  template <typename T>
  static constexpr bool apart = TPR == 0 || CH * Piece<T>::N > 16 || (TPR > 512 && CH > 1);
};
// Calls f(Split) for the lanes and pieces of a row of `width`, f(Split<0, 0>) where no split holds it or it is less than a piece.
// Backward, 129 to 256 pieces, 256 lanes of one against 64 of four: 65536 rows of 2048 bf16 features 145 and 262 us; fp32, whose
// pieces have half as many elements to sum, 100000 rows of 516 features 128 and 117, 65536 of 1024 141 and 152, 3001 of 1001 15.0 and 14.8.
template <typename T, bool BWD, typename F>
auto split_of(int32_t width, F f) {
  const int pieces = (width + Piece<T>::N - 1) / Piece<T>::N;
  if (width < Piece<T>::N) return f(Split<0, 0>{});
  if (pieces <= 8) return f(Split<8, 1>{});
  if (pieces <= 16) return f(Split<16, 1>{});
  if (pieces <= 32) return f(Split<32, 1>{});
  if (pieces <= 64) return f(Split<64, 1>{});
  if (pieces <= 128) return f(Split<64, 2>{});
  if constexpr (!BWD || sizeof(T) == 4)
    if (pieces <= 256) return f(Split<64, 4>{});
  if constexpr (BWD && sizeof(T) == 2)
    if (pieces <= 256) return f(Split<256, 1>{});
  if (pieces <= 512) return f(Split<256, 2>{});
  if constexpr (BWD && sizeof(T) == 2)   // 5120 features: 204 us with two pieces on 512 lanes, 170 so
    if (pieces <= 1024) return f(Split<1024, 1>{});
  if constexpr (!BWD || sizeof(T) == 4)
    if (pieces <= 1024) return f(Split<512, 2>{});
  if (pieces <= 2048) return f(Split<512, 4>{});
  if constexpr (sizeof(T) == 4)
    if (pieces <= 4096) return f(Split<1024, 4>{});
  return f(Split<0, 0>{});
}

// Workgroups of a pass: as many as hold all rows, at most `most` per unit
template <int TPR>
int64_t groups(int64_t rows, int units, int most) {
  const int64_t need = (rows + Shape<TPR>::kRows - 1) / Shape<TPR>::kRows;
  const int64_t fit = (int64_t)units * (TPR > 256 ? 2 : most);
  return need < 1 ? 1 : need < fit ? need : fit;   // no rows: one, which sets the gradients to 0
}
constexpr int kFwdPerUnit = 8;
// Backward, workgroups per unit: two where the lanes have work, more where many of them lie behind the row's end and the loads under way are
// fewer for it (256 MiB a tensor: 2048 bf16 features 145 us with two, 151 with three; 768: 158, 151; 320: 194, 164, with four 150).  fp32 rows
// on four pieces a lane have room for two (768: 155, with three 173).
template <typename T, typename S>
int bwd_per_unit(int32_t width) {
  const int pieces = (width + Piece<T>::N - 1) / Piece<T>::N, lanes = S::tpr * S::ch;
  if (S::ch == 1 && pieces * 20 <= lanes * 13) return 4;
  return pieces * 5 <= lanes * 4 && (sizeof(T) == 2 || S::ch < 4) ? 3 : 2;
}

template <typename S, typename K>
void launch_rows(const LayerNormParams& p, int units, int most, hipStream_t s, K fits, K whole, K ragged, int piece) {
  hipLaunchKernelGGL(p.width == S::tpr * S::ch * piece ? fits : p.width % piece == 0 ? whole : ragged, dim3((unsigned)groups<S::tpr>(p.rows, units, most)), dim3(Shape<S::tpr>::kThreads), 0,
                     s, p);
}

template <typename T>
hipError_t fwd(const LayerNormParams& p, int units, hipStream_t s) {
  return split_of<T, false>(p.width, [&](auto split) {
    using S = decltype(split);
    if constexpr (S::tpr == 0)
      hipLaunchKernelGGL(layer_norm_wide_fwd_kernel<T>, dim3((unsigned)groups<kWideThreads>(p.rows, units, 1)), dim3(kWideThreads), 0, s, p);
    else
      launch_rows<S>(p, units, kFwdPerUnit, s, layer_norm_fwd_kernel<T, S::tpr, S::ch, kFits>, layer_norm_fwd_kernel<T, S::tpr, S::ch, kWhole>,
                     layer_norm_fwd_kernel<T, S::tpr, S::ch, kRagged>, Piece<T>::N);
    return hipGetLastError();
  });
}

template <typename T>
int64_t partials(int64_t rows, int32_t width, int units) {
  return split_of<T, true>(width, [&](auto split) -> int64_t {
    using S = decltype(split);
    if constexpr (S::template apart<T>) return rows < 1 ? 1 : rows < 64 * kWideRows ? (rows + kWideRows - 1) / kWideRows : 64;
    const int64_t g = groups<S::tpr == 0 ? 64 : S::tpr>(rows, units, bwd_per_unit<T, S>(width));
    return g > 1 ? g : 0;
  });
}

template <typename T>
hipError_t bwd(const LayerNormParams& p, int units, hipStream_t s) {
  const bool sums = p.d_weight != nullptr || p.d_bias != nullptr;
  const int64_t count = partials<T>(p.rows, p.width, units);
  hipError_t e = split_of<T, true>(p.width, [&](auto split) {
    using S = decltype(split);
    constexpr bool APART = S::template apart<T>;
    if (APART && sums)   // first: dx may take dy's place
      hipLaunchKernelGGL(layer_norm_wide_columns_kernel<T>, dim3((unsigned)((p.width + kWideCols * Piece<T>::N - 1) / (kWideCols * Piece<T>::N)), (unsigned)count),
                         dim3(kWideCols * kWideRows), 0, s, p);
    if constexpr (S::tpr == 0)
      hipLaunchKernelGGL(layer_norm_wide_bwd_kernel<T>, dim3((unsigned)groups<kWideThreads>(p.rows, units, 1)), dim3(kWideThreads), 0, s, p);
    else
      launch_rows<S>(p, units, bwd_per_unit<T, S>(p.width), s, layer_norm_bwd_kernel<T, S::tpr, S::ch, kFits, !APART>,
                     layer_norm_bwd_kernel<T, S::tpr, S::ch, kWhole, !APART>, layer_norm_bwd_kernel<T, S::tpr, S::ch, kRagged, !APART>, Piece<T>::N);
    return hipGetLastError();
  });
  if (e != hipSuccess || !sums || count == 0) return e;
  return launch_column_sums(p.partial, count, 2 * (int64_t)p.width, p.width, p.d_weight, p.d_bias, s);
}

}  // namespace

// 16 columns a workgroup, 64 threads each; `from`: the launch's first column
constexpr int kSumCols = 16, kSumSlices = 64;
constexpr int64_t kSumMost = 1 << 25;   // columns of a launch: a grid has at most 2^32 - 1 work-items
__global__ __launch_bounds__(kSumCols * kSumSlices) void column_sum_kernel(const float* partial, int64_t count, int64_t columns, int64_t first,
                                                                           int64_t from, float* a, float* b) {
  __shared__ float part[kSumSlices][kSumCols + 1];
  const int col = threadIdx.x % kSumCols, slice = threadIdx.x / kSumCols;
  const int64_t j = from + (int64_t)blockIdx.x * kSumCols + col;
  float v = 0.f;
  if (j < columns) {
#pragma unroll 8
    for (int64_t r = slice; r < count; r += kSumSlices) v += partial[r * columns + j];
  }
  part[slice][col] = v;
  __syncthreads();
  if (slice != 0 || j >= columns) return;
  v = 0.f;
#pragma unroll 16
  for (int i = 0; i < kSumSlices; i++) v += part[i][col];
  if (j < first) {
    if (a != nullptr) a[j] = v;
  } else if (b != nullptr) {
    b[j - first] = v;
  }
}
hipError_t launch_column_sums(const float* partial, int64_t count, int64_t columns, int64_t first, float* a, float* b, hipStream_t s) {
  for (int64_t from = 0; from < columns; from += kSumMost) {
    const int64_t n = columns - from < kSumMost ? columns - from : kSumMost;
    hipLaunchKernelGGL(column_sum_kernel, dim3((unsigned)((n + kSumCols - 1) / kSumCols)), dim3(kSumCols * kSumSlices), 0, s, partial, count, columns,
                       first, from, a, b);
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
  }
  return hipSuccess;
}

hipError_t launch_layer_norm_fwd(int dtype, const LayerNormParams& p, int units, hipStream_t s) {
  if (dtype == kBF16) return fwd<__bf16>(p, units, s);
  if (dtype == kF16) return fwd<_Float16>(p, units, s);
  return fwd<float>(p, units, s);
}

hipError_t launch_layer_norm_bwd(int dtype, const LayerNormParams& p, int units, hipStream_t s) {
  if (dtype == kBF16) return bwd<__bf16>(p, units, s);
  if (dtype == kF16) return bwd<_Float16>(p, units, s);
  return bwd<float>(p, units, s);
}

int64_t layer_norm_bwd_partials(int dtype, int64_t rows, int32_t width, int units) {
  return dtype == kF32 ? partials<float>(rows, width, units) : partials<__bf16>(rows, width, units);
}

}  // namespace la2
