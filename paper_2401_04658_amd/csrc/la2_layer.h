// Internal declarations of the operators around the recurrence (not part of the C ABI): layer normalisation, matrix products
// with an epilogue, beam selection and reordering.
#ifndef LA2_LAYER_H_
#define LA2_LAYER_H_

#include <hip/hip_runtime.h>
#include <stdint.h>

#include <type_traits>

#include "la2_internal.h"

namespace la2 {

// Sixteen bytes of a row, at any address that is a multiple of the element's size (the hardware takes unaligned vector loads
// and stores of global memory).
template <typename T>
struct Piece {
  static constexpr int N = 16 / (int)sizeof(T);
  typedef T vec __attribute__((ext_vector_type(16 / sizeof(T))));
  typedef vec at_element __attribute__((aligned(sizeof(T))));

  // elements at .. at + N - 1 (at a multiple of N) of a row of `width` elements, 0 behind its end: there the row's last N elements, moved
  // down (one load instead of up to N)
  static __device__ __forceinline__ vec raw(const T* row, int64_t at, int64_t width) {
    typedef unsigned __int128 bits;
    if (at + N <= width) return *reinterpret_cast<const at_element*>(row + at);
    bits u = 0;
    if (at < width) {
      if (width >= N) {
        const vec last = *reinterpret_cast<const at_element*>(row + width - N);
        u = __builtin_bit_cast(bits, last) >> (8 * (int)sizeof(T) * (int)(at + N - width));
      } else {
#pragma clang loop unroll(disable)
        for (int i = 0; i < (int)width; i++) {
          typedef std::conditional_t<sizeof(T) == 2, uint16_t, uint32_t> word;
          u |= (bits)reinterpret_cast<const word*>(row)[i] << (8 * (int)sizeof(T) * i);
        }
      }
    }
    return __builtin_bit_cast(vec, u);
  }
  static __device__ __forceinline__ void load(const T* row, int at, int width, float (&v)[N]) {
    const vec u = raw(row, at, width);
#pragma unroll
    for (int i = 0; i < N; i++) v[i] = (float)u[i];
  }
  // `past`: past the caches (whole pieces)
  static __device__ __forceinline__ void store(T* row, int at, int width, const float (&v)[N], bool past = false) {
    vec u;
#pragma unroll
    for (int i = 0; i < N; i++) u[i] = (T)v[i];
    if (at + N <= width) {
      if (past) __builtin_nontemporal_store(u, reinterpret_cast<at_element*>(row + at));
      else *reinterpret_cast<at_element*>(row + at) = u;
    } else if (at < width) {   // halves, quarters, ... of what is left
      typedef unsigned __int128 bits;
      bits b = __builtin_bit_cast(bits, u);
      const int left = width - at;
      T* to = row + at;
#pragma unroll
      for (int n = N / 2; n > 0; n >>= 1) {
        if (left & n) {
          typedef uint64_t u64 __attribute__((aligned(2)));
          typedef uint32_t u32 __attribute__((aligned(2)));
          if (n * sizeof(T) == 8) *reinterpret_cast<u64*>(to) = (uint64_t)b;
          else if (n * sizeof(T) == 4) *reinterpret_cast<u32*>(to) = (uint32_t)b;
          else *reinterpret_cast<uint16_t*>(to) = (uint16_t)b;
          b >>= 8 * (int)sizeof(T) * n;
          to += n;
        }
      }
    }
  }
};

// A lane's piece of rows of one width (a piece at least), fetched in one step and made up in another, so that the load can be under way in
// between.  Lanes behind the row's end and the one across it load what is there: a branch around a load would make the loads behind
// it wait (rows of 200 bf16 features, 256 MiB a tensor, backward: 250 us with one, 148 without).
enum Edge { kFits, kWhole, kRagged };   // rows that the lanes' pieces cover exactly; of whole pieces; of any length
template <typename T, Edge EDGE>
struct RowPiece {
  using P = Piece<T>;
  static constexpr int N = P::N;
  int at, width;
  __device__ __forceinline__ RowPiece(int at_, int width_) : at(at_), width(width_) {}
  __device__ __forceinline__ typename P::vec fetch(const T* row) const {
    return *reinterpret_cast<const typename P::at_element*>(row + (EDGE == kFits ? at : min(at, width - N)));
  }
  __device__ __forceinline__ typename P::vec settle(typename P::vec u) const {
    typedef unsigned __int128 bits;
    if (EDGE == kFits) return u;
    if (EDGE == kWhole) {
      typedef __attribute__((ext_vector_type(4))) uint32_t u32x4;
      u32x4 b = __builtin_bit_cast(u32x4, u);
#pragma unroll
      for (int i = 0; i < 4; i++) b[i] = at < width ? b[i] : 0;
      return __builtin_bit_cast(typename P::vec, b);
    }
    if (at + N > width) {
      bits b = __builtin_bit_cast(bits, u);
      b = at < width ? b >> (8 * (int)sizeof(T) * (at + N - width)) : 0;
      u = __builtin_bit_cast(typename P::vec, b);
    }
    return u;
  }
  __device__ __forceinline__ void store(T* row, const float (&v)[N]) const {
    if (EDGE == kRagged) {
      P::store(row, at, width, v);
    } else if (EDGE == kFits || at < width) {
      typename P::vec u;
#pragma unroll
      for (int i = 0; i < N; i++) u[i] = (T)v[i];
      *reinterpret_cast<typename P::at_element*>(row + at) = u;
    }
  }
};

// A value that the compiler takes for new: what was formed from the old one is formed again rather than kept in registers.
template <typename T>
__device__ __forceinline__ T renewed(T x) {
  if constexpr (std::is_integral_v<T>) asm volatile("" : "+s"(x));
  else asm volatile("" : "+v"(x));
  return x;
}

// N floats of a vector of `width` from element `at` (a multiple of 4) on, `other` behind its end and for a vector that is not given.  The
// vector starts at a multiple of 16 bytes.  WHOLE: its width is a multiple of N, as `at` is.
template <int N, bool WHOLE = false>
__device__ __forceinline__ void load_floats(const float* p, int64_t at, int64_t width, float other, float (&v)[N]) {
  typedef __attribute__((ext_vector_type(4))) float f4;
  if (p != nullptr && at + N <= width) {
#pragma unroll
    for (int i = 0; i < N; i += 4) {
      const f4 u = *reinterpret_cast<const f4*>(p + at + i);
#pragma unroll
      for (int k = 0; k < 4; k++) v[i + k] = u[k];
    }
  } else {
#pragma unroll
    for (int i = 0; i < N; i++) v[i] = !WHOLE && p != nullptr && at + i < width ? p[at + i] : other;
  }
}

// The same from any float on, 0 behind the end
template <int N>
__device__ __forceinline__ void load_any_floats(const float* p, int64_t at, int64_t width, float (&v)[N]) {
#pragma unroll
  for (int i = 0; i < N; i += 4) {
    const auto u = Piece<float>::raw(p, at + i, width);
#pragma unroll
    for (int k = 0; k < 4; k++) v[i + k] = u[k];
  }
}

// ... and their way back; the vector may start at any float
template <int N>
__device__ __forceinline__ void store_floats(float* p, int64_t at, int64_t width, const float (&v)[N]) {
  typedef __attribute__((ext_vector_type(4))) float f4;
  typedef f4 at_float __attribute__((aligned(4)));
  if (at + N <= width) {
#pragma unroll
    for (int i = 0; i < N; i += 4) *reinterpret_cast<at_float*>(p + at + i) = f4{v[i], v[i + 1], v[i + 2], v[i + 3]};
  } else {
#pragma unroll
    for (int i = 0; i < N; i++)
      if (at + i < width) p[at + i] = v[i];
  }
}

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
// a[j] and, from j = first on, b[j - first] = the sums of columns j over `count` rows of partial, in a fixed order
hipError_t launch_column_sums(const float* partial, int64_t count, int64_t columns, int64_t first, float* a, float* b, hipStream_t s);
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
  int32_t chunks, parts;      // workgroups of a row, and parts of the vocabulary that each works off
  uint64_t* keys;             // workspace: [batch * beams][chunks][beams]
  float2* sums;               // workspace: [batch * beams][chunks] (largest logit, sum of exp against it)
  float* out_scores;
  int32_t* parent;
  int32_t* token;
  uint8_t* out_finished;
};
int beam_select_chunks(int64_t rows, int32_t beams, int32_t vocab, int units);
hipError_t launch_beam_select(int dtype, BeamSelectParams p, int units, hipStream_t s);   // sets chunks and parts

constexpr int kMaxStatesPerLaunch = 64;
constexpr int kReorderThreads = 256;   // 16 bytes of a state each
// a grid has at most 2^32 - 1 work-items
constexpr int64_t kMostReorderBytes = (((int64_t)1 << 32) / kReorderThreads - 1) * kReorderThreads * 16;
struct BeamReorderParams {
  int32_t batch, beams;
  int64_t row_bytes;
  const int32_t* parent;
  void* states[kMaxStatesPerLaunch];
};
hipError_t launch_beam_reorder(const BeamReorderParams& p, int nstates, hipStream_t s);

}  // namespace la2
#endif
