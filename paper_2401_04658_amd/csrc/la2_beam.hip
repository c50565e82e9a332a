// Beam search: the best continuations of a batch's beams, and the states that move with them.
//
// Selection.  Candidate (beam i, token t) has the score  s_i + log_softmax(x_i)_t;  the `beams` best of a batch row's beams * vocab
// candidates are taken, equal ones in the order of (beam, token).  Within a beam the order is that of the logits, so the logits are
// read once: a workgroup keeps a piece of a beam's vocabulary in registers and leaves its `beams` largest logits with their
// tokens and its part of the softmax's sum; a second launch, one workgroup per batch row, joins the sums, scores those candidates
// in 64 bits (so that a rounding makes no two of them equal) and takes the best.
//
// Both launches find the n largest the same way: the n-th largest of the threads' own maxima is a bound that at least n values
// reach; the values that reach it (n or a few more, never more than n threads hold) go to LDS, where each one's rank is
// the number of larger ones.  Order and result do not depend on the order in which threads arrive.
#include "la2_layer.h"

namespace la2 {
namespace {

constexpr int kSelectThreads = 256;

// A logit as what it counts for: NaN is no candidate, +inf is the largest finite value, the two zeros are one value.
__device__ __forceinline__ float clean_logit(float x) {
  if (x != x) return -INFINITY;
  return fminf(x, 3.40282346638528859812e38f) + 0.f;
}

// Unsigned number in the order of the floats, and back.
__device__ __forceinline__ uint32_t ordered(float x) {
  const uint32_t u = __float_as_uint(x);
  return u & 0x80000000u ? ~u : u | 0x80000000u;
}
__device__ __forceinline__ float from_ordered(uint32_t u) { return __uint_as_float(u & 0x80000000u ? u & 0x7FFFFFFFu : ~u); }
// Larger logits first, then lower tokens; 0: no candidate.
__device__ __forceinline__ uint64_t key_of(float x, int token) {
  return x == -INFINITY ? 0 : (uint64_t)ordered(x) << 32 | (0xFFFFFFFFu - (uint32_t)token);
}

// Workgroup (chunk, row): the candidates of P * 256 pieces of the row's vocabulary.
template <typename T, int P>
__global__ __launch_bounds__(kSelectThreads) void beam_chunk_kernel(BeamSelectParams p) {
  constexpr int N = Piece<T>::N, W = kSelectThreads / 64;
  __shared__ uint64_t top[kSelectThreads];
  __shared__ uint64_t found[kMaxBeams * P * N];
  __shared__ float red[2][W];
  __shared__ uint64_t bound;
  __shared__ int count;
  const int row = blockIdx.y, n = p.beams, tid = threadIdx.x;
  const int64_t at = (int64_t)row * p.chunks + blockIdx.x;
  if ((p.finished != nullptr && p.finished[row] != 0) || !(p.scores[row] > -INFINITY)) return;   // nothing of it is read
  const T* x = static_cast<const T*>(p.logits) + (int64_t)row * p.stride;
  const int first = blockIdx.x * kSelectThreads * P * N;
  float v[P][N], m = -INFINITY;
  uint64_t best = 0;
#pragma unroll
  for (int c = 0; c < P; c++) Piece<T>::load(x, first + (c * kSelectThreads + tid) * N, p.vocab, v[c]);
#pragma unroll
  for (int c = 0; c < P; c++)
#pragma unroll
    for (int i = 0; i < N; i++) {
      const int token = first + (c * kSelectThreads + tid) * N + i;
      v[c][i] = token < p.vocab ? clean_logit(v[c][i]) : -INFINITY;
      if (v[c][i] > m) {
        m = v[c][i];
        best = key_of(m, token);
      }
    }
  top[tid] = best;
  float all = m;
#pragma unroll
  for (int k = 1; k < 64; k <<= 1) all = fmaxf(all, __shfl_xor(all, k));
  if ((tid & 63) == 0) red[0][tid >> 6] = all;
  if (tid == 0) {
    count = 0;
    bound = 0;
  }
  __syncthreads();
  all = red[0][0];
#pragma unroll
  for (int w = 1; w < W; w++) all = fmaxf(all, red[0][w]);
  float sum = 0.f;
  if (all > -INFINITY) {
#pragma unroll
    for (int c = 0; c < P; c++)
#pragma unroll
      for (int i = 0; i < N; i++) sum += __expf(v[c][i] - all);
  }
#pragma unroll
  for (int k = 1; k < 64; k <<= 1) sum += __shfl_xor(sum, k);
  if ((tid & 63) == 0) red[1][tid >> 6] = sum;
  // the n-th largest of the threads' maxima
  if (best != 0) {
    int larger = 0;
#pragma unroll 8
    for (int k = 0; k < kSelectThreads; k++) larger += top[k] > best;
    if (larger == n - 1) bound = best;
  }
  __syncthreads();
  if (tid == 0) {
    sum = 0.f;
    for (int w = 0; w < W; w++) sum += red[1][w];
    p.sums[at] = make_float2(all, sum);
  }
  const uint64_t b = bound;
  if (best != 0 && best >= b) {
#pragma unroll
    for (int c = 0; c < P; c++)
#pragma unroll
      for (int i = 0; i < N; i++) {
        const uint64_t key = key_of(v[c][i], first + (c * kSelectThreads + tid) * N + i);
        if (key != 0 && key >= b) found[atomicAdd(&count, 1)] = key;
      }
  }
  __syncthreads();
  const int have = count;
  uint64_t* out = p.keys + at * n;
  for (int c = tid; c < have; c += kSelectThreads) {
    const uint64_t key = found[c];
    int larger = 0;
    for (int k = 0; k < have; k++) larger += found[k] > key;
    if (larger < n) out[larger] = key;
  }
  for (int c = have + tid; c < n; c += kSelectThreads) out[c] = 0;
}

// A scored candidate; larger scores first, then the lower place.
struct Scored {
  double score;
  uint32_t place;   // beam * vocab + token
};
__device__ __forceinline__ bool before(const Scored& a, const Scored& b) { return a.score > b.score || (a.score == b.score && a.place < b.place); }

constexpr int kMergeFound = 4096;

// Workgroup per batch row: joins its beams' pieces.
template <int THREADS>
__global__ __launch_bounds__(THREADS) void beam_merge_kernel(BeamSelectParams p) {
  __shared__ double log_sum[kMaxBeams], base[kMaxBeams];   // log of the sum of exp(x - largest), and the largest
  __shared__ int kind[kMaxBeams];                          // 0: no candidates, 1: its vocabulary, 2: finished, one candidate
  __shared__ double top_score[THREADS];
  __shared__ uint32_t top_place[THREADS];
  __shared__ double found_score[kMergeFound];
  __shared__ uint32_t found_place[kMergeFound];
  __shared__ Scored bound;
  __shared__ int count;
  const int n = p.beams, tid = threadIdx.x;
  const int64_t row0 = (int64_t)blockIdx.x * n;
  {   // eight lanes a beam
    const int beam = tid / 8, lane = tid % 8;
    float m = -INFINITY;
    int what = 0;
    if (beam < n) {
      const float s = p.scores[row0 + beam];
      what = !(s > -INFINITY) ? 0 : p.finished != nullptr && p.finished[row0 + beam] != 0 ? 2 : 1;
    }
    const float2* sums = p.sums + (row0 + beam) * p.chunks;
    if (what == 1)
      for (int c = lane; c < p.chunks; c += 8) m = fmaxf(m, sums[c].x);
#pragma unroll
    for (int k = 1; k < 8; k <<= 1) m = fmaxf(m, __shfl_xor(m, k));
    double s = 0.0;
    if (what == 1 && m > -INFINITY)
      for (int c = lane; c < p.chunks; c += 8) s += (double)sums[c].y * exp((double)sums[c].x - (double)m);
#pragma unroll
    for (int k = 1; k < 8; k <<= 1) s += __shfl_xor(s, k);
    if (lane == 0 && beam < n) {
      kind[beam] = what == 1 && !(m > -INFINITY) ? 0 : what;
      base[beam] = (double)m;
      log_sum[beam] = what == 1 && m > -INFINITY ? log(s) : 0.0;
    }
  }
  if (tid == 0) {
    count = 0;
    bound.score = -INFINITY;
    bound.place = 0xFFFFFFFFu;
  }
  __syncthreads();
  const int per = p.chunks * n, total = n * per;
  // candidate c of the row: score -inf for none
  auto candidate = [&](int c) {
    Scored r{-INFINITY, 0xFFFFFFFFu};
    const int beam = c / per, rest = c % per;
    if (kind[beam] == 1) {
      const uint64_t key = p.keys[(row0 + beam) * per + rest];
      if (key != 0) {
        r.score = (double)p.scores[row0 + beam] + (((double)from_ordered((uint32_t)(key >> 32)) - base[beam]) - log_sum[beam]);
        r.place = (uint32_t)beam * (uint32_t)p.vocab + (0xFFFFFFFFu - (uint32_t)key);
      }
    } else if (kind[beam] == 2 && rest == 0) {
      r.score = (double)p.scores[row0 + beam];
      r.place = (uint32_t)beam * (uint32_t)p.vocab + (uint32_t)p.eos;
    }
    return r;
  };
  Scored best{-INFINITY, 0xFFFFFFFFu};
  for (int c = tid; c < total; c += THREADS) {
    const Scored r = candidate(c);
    if (before(r, best)) best = r;
  }
  top_score[tid] = best.score;
  top_place[tid] = best.place;
  __syncthreads();
  if (best.score > -INFINITY) {
    int larger = 0;
#pragma unroll 4
    for (int k = 0; k < THREADS; k++) larger += before(Scored{top_score[k], top_place[k]}, best);
    if (larger == n - 1) bound = best;
  }
  __syncthreads();
  const Scored b = bound;
  if (best.score > -INFINITY && !before(b, best)) {
    for (int c = tid; c < total; c += THREADS) {
      const Scored r = candidate(c);
      if (r.score > -INFINITY && !before(b, r)) {
        const int at = atomicAdd(&count, 1);
        found_score[at] = r.score;
        found_place[at] = r.place;
      }
    }
  }
  __syncthreads();
  const int have = count;
  auto write = [&](int slot, float score, int parent, int token, bool done) {
    p.out_scores[row0 + slot] = score;
    p.parent[row0 + slot] = parent;
    p.token[row0 + slot] = token;
    p.out_finished[row0 + slot] = done ? 1 : 0;
  };
  for (int c = tid; c < have; c += THREADS) {
    const Scored r{found_score[c], found_place[c]};
    int larger = 0;
    for (int k = 0; k < have; k++) larger += before(Scored{found_score[k], found_place[k]}, r);
    if (larger < n) {
      const int parent = (int)(r.place / (uint32_t)p.vocab), token = (int)(r.place % (uint32_t)p.vocab);
      write(larger, (float)r.score, parent, token, kind[parent] == 2 || token == p.eos);
    }
  }
  for (int c = have + tid; c < n; c += THREADS) write(c, -INFINITY, c, p.eos >= 0 ? p.eos : 0, true);
}

// A thread handles the same 16 bytes of all beams of a batch row: it reads what moves, then writes it, so that the states
// change in place whatever the parents are.  Sources that several beams take come from the caches after the first read; a beam that
// is its own parent is not touched.
template <int MAX>
__global__ __launch_bounds__(256) void beam_reorder_kernel(BeamReorderParams p) {
  typedef __attribute__((ext_vector_type(4))) uint32_t u32x4;
  const int64_t at = ((int64_t)blockIdx.x * 256 + threadIdx.x) * 16;
  if (at >= p.row_bytes) return;
  const int32_t* parent = p.parent + (int64_t)blockIdx.y * p.beams;
  char* base = static_cast<char*>(p.states[blockIdx.z]) + (int64_t)blockIdx.y * p.beams * p.row_bytes + at;
  u32x4 v[MAX];
  bool moves[MAX];
#pragma unroll
  for (int j = 0; j < MAX; j++) {
    moves[j] = false;
    if (j < p.beams) {
      const int from = parent[j];
      moves[j] = from != j && from >= 0 && from < p.beams;
      if (moves[j]) v[j] = *reinterpret_cast<const u32x4*>(base + from * p.row_bytes);
    }
  }
#pragma unroll
  for (int j = 0; j < MAX; j++)
    if (moves[j]) *reinterpret_cast<u32x4*>(base + j * p.row_bytes) = v[j];
}

// Pieces per thread of the first launch: large ones where the rows alone fill the device
template <typename T>
int pieces(int64_t rows, int32_t vocab, int units) {
  constexpr int kSmall = 4096 / (kSelectThreads * Piece<T>::N), kLarge = 8192 / (kSelectThreads * Piece<T>::N);
  return vocab > 64 * 4096 || rows * ((vocab + 8191) / 8192) >= 4 * units ? kLarge : kSmall;
}

template <typename T>
hipError_t select(const BeamSelectParams& p, hipStream_t s) {
  constexpr int kSmall = 4096 / (kSelectThreads * Piece<T>::N), kLarge = 8192 / (kSelectThreads * Piece<T>::N);
  const dim3 grid((unsigned)p.chunks, (unsigned)(p.batch * p.beams));
  if ((p.vocab + 4095) / 4096 == p.chunks)
    hipLaunchKernelGGL((beam_chunk_kernel<T, kSmall>), grid, dim3(kSelectThreads), 0, s, p);
  else
    hipLaunchKernelGGL((beam_chunk_kernel<T, kLarge>), grid, dim3(kSelectThreads), 0, s, p);
  hipError_t e = hipGetLastError();
  if (e != hipSuccess) return e;
  // candidates of a batch row: the values that reach the bound have to fit found_*: `beams` threads' shares
  const int64_t total = (int64_t)p.beams * p.chunks * p.beams;
  if (total <= 4096)
    hipLaunchKernelGGL(beam_merge_kernel<256>, dim3((unsigned)p.batch), dim3(256), 0, s, p);
  else
    hipLaunchKernelGGL(beam_merge_kernel<1024>, dim3((unsigned)p.batch), dim3(1024), 0, s, p);
  return hipGetLastError();
}

}  // namespace

// One vocabulary of kMaxVocab tokens has 128 pieces, kMaxBeams of them with kMaxBeams candidates each 131,072 candidates, 128 a thread
// of the second launch: kMaxBeams threads' shares are 4096.
static_assert(kMaxBeams * (kMaxBeams * kMaxBeams * (kMaxVocab / 8192) / 1024) <= kMergeFound, "the second launch's list");
static_assert(kMaxBeams * (4096 / 256) <= kMergeFound, "the second launch's list, 256 threads");
static_assert(64 * kMaxBeams * kMaxBeams / 1024 * kMaxBeams <= kMergeFound, "the second launch's list, small pieces");

int beam_select_chunks(int dtype, int64_t rows, int32_t vocab, int units) {
  const int p = dtype == kF32 ? pieces<float>(rows, vocab, units) * 4 : pieces<__bf16>(rows, vocab, units) * 8;
  const int piece = p * kSelectThreads;
  return (vocab + piece - 1) / piece;
}

hipError_t launch_beam_select(int dtype, const BeamSelectParams& p, hipStream_t s) {
  if (dtype == kBF16) return select<__bf16>(p, s);
  if (dtype == kF16) return select<_Float16>(p, s);
  return select<float>(p, s);
}

hipError_t launch_beam_reorder(const BeamReorderParams& p, int nstates, hipStream_t s) {
  const int64_t threads = p.row_bytes / 16;
  const dim3 grid((unsigned)((threads + 255) / 256), (unsigned)p.batch, (unsigned)nstates);
  if (p.beams <= 4) hipLaunchKernelGGL(beam_reorder_kernel<4>, grid, dim3(256), 0, s, p);
  else if (p.beams <= 8) hipLaunchKernelGGL(beam_reorder_kernel<8>, grid, dim3(256), 0, s, p);
  else if (p.beams <= 16) hipLaunchKernelGGL(beam_reorder_kernel<16>, grid, dim3(256), 0, s, p);
  else hipLaunchKernelGGL(beam_reorder_kernel<32>, grid, dim3(256), 0, s, p);
  return hipGetLastError();
}

}  // namespace la2
