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
size_t linear_fwd_workspace(const LinearParams& p, int units);
size_t linear_bwd_workspace(const LinearParams& p, int units);
hipError_t launch_linear_fwd(const LinearParams& p, void* workspace, int units, hipStream_t s);
hipError_t launch_linear_bwd(const LinearParams& p, void* workspace, int units, hipStream_t s);

enum { kTile64 = 0, kTile128 = 1, kTile256 = 2 };
hipError_t launch_product_bf16(int tile, bool across_a, bool across_b, const ProductParams& p, hipStream_t s);
hipError_t launch_product_f16(int tile, bool across_a, bool across_b, const ProductParams& p, hipStream_t s);
hipError_t launch_product_f32(int tile, bool across_a, bool across_b, const ProductParams& p, hipStream_t s);

// erfc(z) for z >= 0 as exp(-z^2) times a polynomial in 1 / (1 + 0.3275911 z): Abramowitz and Stegun, Handbook of Mathematical
// Functions, 7.1.26 (absolute error 1.5e-7).  `e` = exp(-z^2).
__device__ __forceinline__ float erfc_from(float z, float e) {
  const float t = __builtin_amdgcn_rcpf(fmaf(0.3275911f, z, 1.f));
  float s = fmaf(1.061405429f, t, -1.453152027f);
  s = fmaf(s, t, 1.421413741f);
  s = fmaf(s, t, -0.284496736f);
  s = fmaf(s, t, 0.254829592f);
  return s * t * e;
}
constexpr float kHalfRoot = 0.70710678118654752440f, kLog2e = 1.44269504088896340736f;
// The normal distribution function at x, and exp(-x^2 / 2)
__device__ __forceinline__ float normal_cdf(float x, float& e) {
  const float z = fabsf(x) * kHalfRoot;
  e = __builtin_amdgcn_exp2f(-z * z * kLog2e);
  const float tail = 0.5f * erfc_from(z, e);
  return x < 0.f ? tail : 1.f - tail;
}
__device__ __forceinline__ float sigmoid(float x) { return __builtin_amdgcn_rcpf(1.f + __builtin_amdgcn_exp2f(-x * kLog2e)); }

// act(z) and its slope.  An infinite z keeps the limits: 0 * inf is not formed.
__device__ __forceinline__ float act_of(float z, int act) {
  if (act == kActRelu) return z > 0.f ? z : z == z ? 0.f : z;
  if (act == kActGelu) {
    float e;
    const float c = normal_cdf(z, e);
    return c == 0.f ? 0.f : z * c;
  }
  if (act == kActSilu) {
    const float c = sigmoid(z);
    return c == 0.f ? 0.f : z * c;
  }
  return z;
}
__device__ __forceinline__ float act_slope(float z, int act) {
  if (act == kActRelu) return z > 0.f ? 1.f : z == z ? 0.f : z;
  if (act == kActGelu) {
    float e;
    const float c = normal_cdf(z, e);
    return e == 0.f ? c : fmaf(z * 0.39894228040143267794f, e, c);   // 1 / sqrt(2 pi)
  }
  if (act == kActSilu) {
    const float c = sigmoid(z);
    return c == 0.f ? 0.f : c == 1.f ? 1.f : c * fmaf(z, 1.f - c, 1.f);
  }
  return 1.f;
}

// N sums of row i from column j on, finished: bias, pre, activation, residual, rounded once.
template <typename E, int N>
__device__ __forceinline__ void finish(const ProductParams& p, int64_t i, int64_t j, float (&v)[N]) {
  static_assert(N == Piece<E>::N, "one piece");
  const int64_t row = i * p.ldo;
  if (p.bias != nullptr) {
    float b[N];
    load_floats(p.bias, j, p.J, 0.f, b);
#pragma unroll
    for (int k = 0; k < N; k++) v[k] += b[k];
  }
  if (p.pre != nullptr) Piece<E>::store(static_cast<E*>(p.pre) + row, (int)j, (int)p.J, v);
  if (p.act != kActNone) {
#pragma unroll
    for (int k = 0; k < N; k++) v[k] = act_of(v[k], p.act);
  }
  if (p.residual != nullptr) {
    float r[N];
    Piece<E>::load(static_cast<const E*>(p.residual) + row, (int)j, (int)p.J, r);
#pragma unroll
    for (int k = 0; k < N; k++) v[k] += r[k];
  }
  Piece<E>::store(static_cast<E*>(p.out) + row, (int)j, (int)p.J, v);
}

}  // namespace la2
#endif
