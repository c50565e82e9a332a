// Matrix products with an epilogue: what the translation units of the 16-bit and fp32 types share (not part of the C ABI).
//
//   c[i][j] = sum_r a(i, r) b(j, r)        i < I, j < J, r < R
//
// An operand's rows run either along r ("along": x and w of the forward pass) or along its own index ("across": element (i, r) at
// r * ld + i, as both operands of the weight's gradient and w of the input's).
#ifndef LA2_LINEAR_H_
#define LA2_LINEAR_H_

#include <hip/hip_runtime.h>
#include <stdint.h>

#include "la2_layer.h"

namespace la2 {

enum { kActNone = 0, kActRelu = 1, kActGelu = 2, kActSilu = 3 };

struct ProductParams {
  int64_t I, J, R;
  const void *a, *b;
  int64_t lda, ldb;         // elements between rows
  // epilogue: z = c + bias[j], out = act(z) + residual, pre = z; rows of out, pre and residual are ldo elements apart
  const float* bias;
  const void* residual;
  void* out;
  void* pre;
  int64_t ldo;
  int32_t act;
  int32_t past;   // out and pre go past the caches: too large to be found there by what reads them next
  // The reduction cut into `splits` pieces of `span` (a multiple of the kernels' step): the pieces' sums go to partial
  // [splits][I][J] and a launch of its own joins them.  splits == 1: partial is not used.
  int32_t splits;
  int64_t span;
  float* partial;
};

// What a call is given; the pointers that are not wanted are nullptr.
struct LinearParams {
  int64_t rows;
  int32_t in, out, dtype, act;
  int64_t stride_x, stride_w, stride_y;
  const void *x, *w;
  const float* bias;
  const void* residual;
  void *y, *pre;                 // pre: written by the forward pass, read by the backward pass
  const void* dy;
  void *dx, *dw;
  float* d_bias;
};
// Whether the products' grids stay below the 2^32 work-items that a launch may have, with the largest tile: fewer than 2^23 workgroups of 512
// threads, 2^18 of them set aside for those that sum d_bias.
bool linear_fits(const LinearParams& p);
size_t linear_fwd_workspace(const LinearParams& p, int units);
size_t linear_bwd_workspace(const LinearParams& p, int units);
hipError_t launch_linear_fwd(const LinearParams& p, void* workspace, int units, hipStream_t s);
hipError_t launch_linear_bwd(const LinearParams& p, void* workspace, int units, hipStream_t s);

// Both products of a backward pass (the input's gradient: a along, b across; the weight's: both across) in one launch, workgroups
// [0, first) the one with the longer way, and behind them those that sum the columns of `partial` into d_bias.
struct PairParams {
  ProductParams p[2];        // 0: the input's gradient, 1: the weight's
  int32_t groups[2];         // workgroups of each; 0: not wanted
  int32_t weight_first;
  const float* partial;      // [count][width], nullptr: no sums
  int32_t count, width;
  float* sums;
};

enum { kTile64 = 0, kTile128 = 1, kTile256 = 2, kTiles = 3 };
constexpr int kTileThreads[kTiles] = {256, 256, 512};
constexpr int64_t kMostThreads = ((int64_t)1 << 32) - 1;   // of a grid
constexpr int64_t kMostSumGroups = 1 << 18;                // workgroups that sum d_bias: 16 columns each, rows of less than 2^23 bytes
hipError_t launch_product_bf16(int tile, const ProductParams& p, hipStream_t s);
hipError_t launch_product_f16(int tile, const ProductParams& p, hipStream_t s);
hipError_t launch_product_f32(int tile, const ProductParams& p, hipStream_t s);
hipError_t launch_pair_bf16(int tile, const PairParams& p, hipStream_t s);
hipError_t launch_pair_f16(int tile, const PairParams& p, hipStream_t s);
hipError_t launch_pair_f32(int tile, const PairParams& p, hipStream_t s);

// exp(-x^2 / 2) and the normal distribution's tail Phi(-a) at a = min(|x|, 64), as exp(-z^2) times a polynomial in 1 / (1 + 0.3275911 z), z = a /
// sqrt(2): Abramowitz and Stegun, Handbook of Mathematical Functions, 7.1.26 (absolute error 1.5e-7 of erfc, half of that here).
constexpr float kHalfRoot = 0.70710678118654752440f, kLog2e = 1.44269504088896340736f;
__device__ __forceinline__ float normal_tail(float x, float& a, float& e) {
  a = fminf(fabsf(x), 64.f);
  e = __builtin_amdgcn_exp2f(x * x * (-0.5f * kLog2e));
  const float t = __builtin_amdgcn_rcpf(fmaf(0.3275911f * kHalfRoot, a, 1.f));
  float s = fmaf(0.5f * 1.061405429f, t, 0.5f * -1.453152027f);
  s = fmaf(s, t, 0.5f * 1.421413741f);
  s = fmaf(s, t, 0.5f * -0.284496736f);
  s = fmaf(s, t, 0.5f * 0.254829592f);
  return s * t * e;
}
__device__ __forceinline__ float sigmoid(float x) { return __builtin_amdgcn_rcpf(1.f + __builtin_amdgcn_exp2f(-x * kLog2e)); }

// act(z) and its slope.  Factors that may be infinite are cut where the other factor has become 0; a NaN comes through the other factor.
template <int ACT>
__device__ __forceinline__ float act_of(float z) {
  if (ACT == kActRelu) return z > 0.f ? z : z == z ? 0.f : z;
  if (ACT == kActGelu) {   // z Phi(z) = max(z, 0) - |z| Phi(-|z|)
    float a, e;
    const float tail = normal_tail(z, a, e);
    return fmaf(-a, tail, fmaxf(z, 0.f));
  }
  if (ACT == kActSilu) return fmaxf(z, -2000.f) * sigmoid(z);
  return z;
}
template <int ACT>
__device__ __forceinline__ float act_slope(float z) {
  if (ACT == kActRelu) return z > 0.f ? 1.f : z == z ? 0.f : z;
  if (ACT == kActGelu) {   // Phi(z) + z exp(-z^2 / 2) / sqrt(2 pi)
    float a, e;
    const float tail = normal_tail(z, a, e);
    return fmaf(copysignf(a, z) * 0.39894228040143267794f, e, z < 0.f ? tail : 1.f - tail);
  }
  if (ACT == kActSilu) {
    const float c = sigmoid(z);
    return c * fmaf(fminf(fmaxf(z, -2000.f), 2000.f), 1.f - c, 1.f);
  }
  return 1.f;
}
template <int ACT>
struct Act {
  static constexpr int value = ACT;
};
template <typename F>
__device__ __forceinline__ void with_act(int act, F f) {
  if (act == kActNone) f(Act<kActNone>{});
  else if (act == kActRelu) f(Act<kActRelu>{});
  else if (act == kActGelu) f(Act<kActGelu>{});
  else f(Act<kActSilu>{});
}

// N sums of row i from column j on, finished: bias (b), pre, activation, residual, rounded once.
template <typename E, int ACT, int N>
__device__ __forceinline__ void finish(const ProductParams& p, int64_t i, int64_t j, const float (&b)[N], float (&v)[N]) {
  static_assert(N == Piece<E>::N, "one piece");
  const int64_t row = i * p.ldo;
#pragma unroll
  for (int k = 0; k < N; k++) v[k] += b[k];
  if (p.pre != nullptr) Piece<E>::store(static_cast<E*>(p.pre) + row, (int)j, (int)p.J, v, p.past != 0);
#pragma unroll
  for (int k = 0; k < N; k++) v[k] = act_of<ACT>(v[k]);
  if (p.residual != nullptr) {
    float r[N];
    Piece<E>::load(static_cast<const E*>(p.residual) + row, (int)j, (int)p.J, r);
#pragma unroll
    for (int k = 0; k < N; k++) v[k] += r[k];
  }
  Piece<E>::store(static_cast<E*>(p.out) + row, (int)j, (int)p.J, v, p.past != 0);
}

}  // namespace la2
#endif
