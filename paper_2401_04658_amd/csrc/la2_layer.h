// Internal declarations of the operators around the recurrence (not part of the C ABI): layer normalisation, matrix products
// with an epilogue, beam selection and reordering.
#ifndef LA2_LAYER_H_
#define LA2_LAYER_H_

#include <hip/hip_runtime.h>
#include <stdint.h>

#include "la2_internal.h"

namespace la2 {

// Sixteen bytes of a row, at any address that is a multiple of the element's size (the hardware takes unaligned vector loads
// and stores of global memory).
template <typename T>
struct Piece {
  static constexpr int N = 16 / (int)sizeof(T);
  typedef T vec __attribute__((ext_vector_type(16 / sizeof(T))));
  typedef vec at_element __attribute__((aligned(sizeof(T))));

  // elements at .. at + N - 1 of a row of `width` elements, 0 behind its end
  static __device__ __forceinline__ void load(const T* row, int at, int width, float (&v)[N]) {
    if (at + N <= width) {
      const vec u = *reinterpret_cast<const at_element*>(row + at);
#pragma unroll
      for (int i = 0; i < N; i++) v[i] = (float)u[i];
    } else {
#pragma unroll
      for (int i = 0; i < N; i++) v[i] = at + i < width ? (float)row[at + i] : 0.f;
    }
  }
  static __device__ __forceinline__ void store(T* row, int at, int width, const float (&v)[N]) {
    if (at + N <= width) {
      vec u;
#pragma unroll
      for (int i = 0; i < N; i++) u[i] = (T)v[i];
      *reinterpret_cast<at_element*>(row + at) = u;
    } else {
#pragma unroll
      for (int i = 0; i < N; i++)
        if (at + i < width) row[at + i] = (T)v[i];
    }
  }
};

struct LayerNormParams {
  int64_t rows;
  int32_t width;
  int64_t stride;        // elements between rows of x, dy, y, dx
  const void* x;
  const void* dy;        // backward
  void* y;               // forward: y; backward: dx
  const float* weight;   // nullptr: 1
  const float* bias;     // nullptr: 0
  float eps;
  float* mean;
  float* rstd;
  float* d_weight;       // nullptr: not wanted
  float* d_bias;
  float* partial;        // [workgroups][2][width]
};
hipError_t launch_layer_norm_fwd(int dtype, const LayerNormParams& p, int units, hipStream_t s);
hipError_t launch_layer_norm_bwd(int dtype, const LayerNormParams& p, int units, hipStream_t s);
// rows of partial sums that the backward pass writes; 0: it needs none
int64_t layer_norm_bwd_partials(int dtype, int64_t rows, int32_t width, int units);

constexpr int kMaxBeams = 32;
constexpr int kMaxVocab = 1 << 20;
struct BeamSelectParams {
  int32_t batch, beams, vocab;
  int64_t stride;             // elements between the rows of logits
  const void* logits;         // [batch][beams] rows
  const float* scores;        // [batch][beams]
  const uint8_t* finished;    // [batch][beams] or nullptr
  int32_t eos;                // -1: none
  int32_t chunks;             // pieces of the vocabulary
  uint64_t* keys;             // workspace: [batch * beams][chunks][beams]
  float2* sums;               // workspace: [batch * beams][chunks] (largest logit, sum of exp against it)
  float* out_scores;
  int32_t* parent;
  int32_t* token;
  uint8_t* out_finished;
};
int beam_select_chunks(int dtype, int64_t rows, int32_t vocab, int units);
hipError_t launch_beam_select(int dtype, const BeamSelectParams& p, hipStream_t s);

constexpr int kMaxStatesPerLaunch = 64;
struct BeamReorderParams {
  int32_t batch, beams;
  int64_t row_bytes;
  const int32_t* parent;
  void* states[kMaxStatesPerLaunch];
};
hipError_t launch_beam_reorder(const BeamReorderParams& p, int nstates, hipStream_t s);

}  // namespace la2
#endif
