// Beam search: the best continuations of a batch's beams, and the states that move with them.
//
// Selection.  Candidate (beam i, token t) has the score  s_i + log_softmax(x_i)_t;  the `beams` best of a batch row's beams * vocab
// candidates are taken, equal ones in the order of (beam, token).  Within a beam the order is that of the logits, so the logits are
// read once: a workgroup keeps a piece of a beam's vocabulary in registers and leaves its `beams` largest logits with their
// tokens and its part of the softmax's sum; a second launch, one workgroup per batch row, joins the sums, scores those candidates
// in 64 bits (so that a rounding makes no two of them equal) and takes the best.
//
// The n largest of a piece: the lanes form n groups or a few more; the smallest of the groups' maxima is a bound that at least n values
// reach, and among values in no particular order n (1 + 1/2 + ... + 1/n) or so.  Those go to LDS, where each one's rank is the number of
// larger ones.  Where more reach it than the list holds (many equal values) the n largest are taken one after the other.  The
// candidates of the second launch are lists in order, which makes such a bound a poor one: there a wave's n-th largest of its lanes'
// maxima is found bit by bit, with the lanes' votes, and the largest of the waves' is the bound (at most n lanes of a wave hold
// anything that reaches it).  Order and result do not depend on the order in which threads arrive.
//
// 32 x 8 beams over 50021 fp32 logits: 17 and 5.5 us (51 MB; the pieces' loads alone take 13); 4 beams over 32000 bf16 logits: 5.2 and 4.8, latency.
#include "la2_layer.h"

namespace la2 {
namespace {

constexpr int kSelectThreads = 256;
constexpr int kList = 512;   // values that are ranked at once

// A logit as what it counts for: NaN is no candidate, +inf is the largest finite value.
__device__ __forceinline__ float clean_logit(float x) { return fminf(fmaxf(x, -INFINITY), 3.40282346638528859812e38f); }

// Unsigned numbers in the order of the floating ones, larger than 0 for all but -NaN, and back.
__device__ __forceinline__ uint32_t ordered(float x) {
  const uint32_t u = __float_as_uint(x);
  return u & 0x80000000u ? ~u : u | 0x80000000u;
}
__device__ __forceinline__ float from_ordered(uint32_t u) { return __uint_as_float(u & 0x80000000u ? u & 0x7FFFFFFFu : ~u); }
__device__ __forceinline__ uint64_t ordered(double x) {
  const uint64_t u = (uint64_t)__double_as_longlong(x);
  return u >> 63 ? ~u : u | (uint64_t)1 << 63;
}
__device__ __forceinline__ double from_ordered(uint64_t u) {
  return __longlong_as_double((long long)(u >> 63 ? u & ~((uint64_t)1 << 63) : ~u));
}
// Larger logits first (the two zeros are one), then lower tokens; 0: no candidate.
__device__ __forceinline__ uint64_t key_of(float x, int token) {
  return x == -INFINITY ? 0 : (uint64_t)ordered(x + 0.f) << 32 | (0xFFFFFFFFu - (uint32_t)token);
}

// How many of `have` values are larger than the one that larger(k) compares with value k: eight lanes count together.
constexpr int kRankLanes = 8;
template <typename F>
__device__ __forceinline__ int rank_of(int have, F larger) {
  int n = 0;
#pragma unroll 2
  for (int k = threadIdx.x % kRankLanes; k < have; k += kRankLanes) n += larger(k);
#pragma unroll
  for (int k = 1; k < kRankLanes; k <<= 1) n += __shfl_xor(n, k);
  return n;
}

__device__ __forceinline__ int votes(bool yes) { return __popcll(__ballot(yes)); }

// The largest T that at least n of the `in` lanes' words reach (0 if there are fewer than n), or a smaller one that exactly n reach.
__device__ __forceinline__ uint32_t nth_word(uint32_t word, bool in, int n) {
  uint32_t t = 0;
  for (int bit = 30; bit >= 0; bit -= 2) {   // two bits at a time: the three votes do not wait for one another
    const uint32_t one = t | 1u << bit, two = t | 2u << bit, three = t | 3u << bit;
    const int reach1 = votes(in && word >= one), reach2 = votes(in && word >= two), reach3 = votes(in && word >= three);
    const int reach = reach3 >= n ? reach3 : reach2 >= n ? reach2 : reach1;
    t = reach3 >= n ? three : reach2 >= n ? two : reach1 >= n ? one : t;
    if (reach == n) break;
  }
  return t;
}
// A bound that exactly n of the wave's lanes reach, compared word by word (WORDS of them, the highest first); all words 0 if fewer than n
// lanes have anything.  The lanes' words differ from one another where they are not 0.
template <int WORDS>
__device__ __forceinline__ void wave_bound(const uint32_t (&word)[WORDS], int n, uint32_t (&bound)[WORDS]) {
  bool in = word[0] != 0;
#pragma unroll
  for (int k = 0; k < WORDS; k++) bound[k] = 0;
  if (votes(in) < n) return;
#pragma unroll
  for (int k = 0; k < WORDS; k++) {
    bound[k] = nth_word(word[k], in, n);
    if (votes(in && word[k] >= bound[k]) == n) return;   // everything from here on
    n -= votes(in && word[k] > bound[k]);
    in = in && word[k] == bound[k];
  }
}

// Workgroup (row, chunk): the largest of `parts` times P * 256 pieces of the row's vocabulary.
template <typename T, int P>
__global__ __launch_bounds__(kSelectThreads) void beam_chunk_kernel(BeamSelectParams p) {
  constexpr int N = Piece<T>::N, PART = kSelectThreads * P * N, WAVES = kSelectThreads / 64;
  __shared__ uint64_t found[kList + kMaxBeams];
  __shared__ uint64_t best_of[kMaxBeams];   // of the parts so far, in their order
  __shared__ uint64_t round_best[2][WAVES];
  __shared__ float high[WAVES][32], part_sum[WAVES];
  __shared__ int count;
  const int row = blockIdx.x / p.chunks, n = p.beams, tid = threadIdx.x, wave = tid >> 6, lane = tid & 63;
  if ((p.finished != nullptr && p.finished[row] != 0) || !(p.scores[row] > -INFINITY)) return;   // nothing of it is read
  const int groups = n <= 4 ? 4 : n <= 8 ? 8 : n <= 16 ? 16 : 32;   // lanes of one number modulo this
  const T* x = static_cast<const T*>(p.logits) + (int64_t)row * p.stride;
  const int begin = blockIdx.x % p.chunks * (p.parts * PART);
  const int end = min(p.vocab, begin + p.parts * PART);
  float largest = -INFINITY, total = 0.f;   // of the parts so far
  int kept = 0;
  for (int first = begin; first < end; first += PART) {
    float v[P][N], m = -INFINITY, second = -INFINITY;   // a thread's largest two
    typename Piece<T>::vec raw[P];
    if (p.vocab >= N) {
#pragma unroll
      for (int c = 0; c < P; c++) raw[c] = RowPiece<T, kRagged>(first + (c * kSelectThreads + tid) * N, p.vocab).fetch(x);
#pragma unroll
      for (int c = 0; c < P; c++) raw[c] = RowPiece<T, kRagged>(first + (c * kSelectThreads + tid) * N, p.vocab).settle(raw[c]);
    } else {
#pragma unroll
      for (int c = 0; c < P; c++) raw[c] = Piece<T>::raw(x, first + (c * kSelectThreads + tid) * N, p.vocab);
    }
    if (tid == 0) count = 0;
#pragma unroll
    for (int c = 0; c < P; c++) {
      const int at = first + (c * kSelectThreads + tid) * N;
      if (at + N <= p.vocab) {
#pragma unroll
        for (int i = 0; i < N; i++) v[c][i] = clean_logit((float)raw[c][i]);
      } else {
#pragma unroll
        for (int i = 0; i < N; i++) v[c][i] = at + i < p.vocab ? clean_logit((float)raw[c][i]) : -INFINITY;
      }
#pragma unroll
      for (int i = 0; i < N; i++) {
        second = __builtin_amdgcn_fmed3f(m, second, v[c][i]);
        m = fmaxf(m, v[c][i]);
      }
    }
    float all = m;
    for (int k = 32; k >= groups; k >>= 1) all = fmaxf(all, __shfl_xor(all, k));
    if (lane < groups) high[wave][lane] = all;
    __syncthreads();
    all = high[0][lane % groups];
#pragma unroll
    for (int w = 1; w < WAVES; w++) all = fmaxf(all, high[w][lane % groups]);
    float bound = all;
    for (int k = 1; k < groups; k <<= 1) {
      all = fmaxf(all, __shfl_xor(all, k));
      bound = fminf(bound, __shfl_xor(bound, k));
    }
    if (kept == n) bound = fmaxf(bound, from_ordered((uint32_t)(best_of[n - 1] >> 32)));
    if (m > -INFINITY && m >= bound) {
      int at = 0;   // the first of the thread's largest
#pragma unroll
      for (int c = P - 1; c >= 0; c--)
#pragma unroll
        for (int i = N - 1; i >= 0; i--) at = v[c][i] == m ? c * N + i : at;
      const int to = atomicAdd(&count, 1);
      if (to < kList) found[to] = key_of(m, first + (at / N * kSelectThreads + tid) * N + at % N);
      if (second > -INFINITY && second >= bound) {
#pragma unroll
        for (int c = 0; c < P; c++)
#pragma unroll
          for (int i = 0; i < N; i++)
            if (v[c][i] > -INFINITY && v[c][i] >= bound && c * N + i != at) {
              const int to = atomicAdd(&count, 1);
              if (to < kList) found[to] = key_of(v[c][i], first + (c * kSelectThreads + tid) * N + i);
            }
      }
    }
    float sum = 0.f;
    if (all > -INFINITY) {
#pragma unroll
      for (int c = 0; c < P; c++)
#pragma unroll
        for (int i = 0; i < N; i++) sum += __expf(v[c][i] - all);
#pragma unroll
      for (int k = 1; k < 64; k <<= 1) sum += __shfl_xor(sum, k);
    }
    if (lane == 0) part_sum[wave] = sum;
    __syncthreads();
    if (all > -INFINITY) {
      sum = 0.f;
#pragma unroll
      for (int w = 0; w < WAVES; w++) sum += part_sum[w];
      const float top = fmaxf(all, largest);
      total = total * (largest > -INFINITY ? __expf(largest - top) : 0.f) + sum * __expf(all - top);
      largest = top;
    }
    const int fresh = count;
    if (fresh <= kList) {
      if (tid < kept) found[fresh + tid] = best_of[tid];
      __syncthreads();
      const int have = fresh + kept;
      for (int c = tid / kRankLanes; c < have; c += kSelectThreads / kRankLanes) {
        const uint64_t key = found[c];
        const int rank = rank_of(have, [&](int k) { return found[k] > key; });
        if (rank < n && tid % kRankLanes == 0) best_of[rank] = key;
      }
      kept = min(n, have);
    } else {   // one after the other
      const uint64_t before = tid < kept ? best_of[tid] : 0;
      uint64_t last = ~(uint64_t)0;
      for (kept = 0; kept < n; kept++) {
        uint64_t best = before < last ? before : 0;
#pragma unroll
        for (int c = 0; c < P; c++)
#pragma unroll
          for (int i = 0; i < N; i++) {
            const uint64_t key = key_of(v[c][i], first + (c * kSelectThreads + tid) * N + i);
            best = key < last && key > best ? key : best;
          }
#pragma unroll
        for (int k = 1; k < 64; k <<= 1) {
          const uint64_t other = __shfl_xor((unsigned long long)best, k);
          best = other > best ? other : best;
        }
        if (lane == 0) round_best[kept & 1][wave] = best;
        __syncthreads();
        last = 0;
#pragma unroll
        for (int w = 0; w < WAVES; w++) last = round_best[kept & 1][w] > last ? round_best[kept & 1][w] : last;
        if (last == 0) break;   // (more than kList values: there are n)
        if (tid == 0) best_of[kept] = last;
      }
    }
    __syncthreads();
  }
  const int64_t to = (int64_t)blockIdx.x;   // row * chunks + chunk
  if (tid == 0) p.sums[to] = make_float2(largest, total);
  if (tid < n) p.keys[to * n + tid] = tid < kept ? best_of[tid] : 0;
}

// Workgroup per batch row: joins its beams' pieces, up to KPT candidates a thread.
template <int THREADS, int KPT>
__global__ __launch_bounds__(THREADS) void beam_merge_kernel(BeamSelectParams p) {
  constexpr int WAVES = THREADS / 64;
  __shared__ double log_sum[kMaxBeams], base[kMaxBeams];   // log of the sum of exp(x - largest), and the largest
  __shared__ float start[kMaxBeams];
  __shared__ int kind[kMaxBeams];                          // 0: no candidates, 1: its vocabulary, 2: finished, one candidate
  __shared__ uint32_t bounds[WAVES][3];
  struct __align__(16) Scored {
    uint64_t score;
    uint32_t place;
  };
  __shared__ Scored found[kMaxBeams * WAVES * KPT];   // at most n lanes a wave hold any
  __shared__ int count;
  const int n = p.beams, tid = threadIdx.x;
  const int64_t row0 = (int64_t)blockIdx.x * n;
  const int per = p.chunks * n, total = n * per;
  uint64_t key[KPT];
#pragma unroll
  for (int k = 0; k < KPT; k++) {   // (those of finished and dead beams were not written and are not used)
    const int c = tid + k * THREADS;
    const uint64_t there = p.keys[row0 * per + min(c, total - 1)];   // (no branch: the loads are all under way together)
    key[k] = c < total ? there : 0;
  }
  if (tid < 8 * kMaxBeams) {   // eight lanes a beam
    const int beam = tid / 8, lane = tid % 8;
    float m = -INFINITY, s0 = -INFINITY;
    int what = 0;
    if (beam < n) {
      s0 = p.scores[row0 + beam];
      what = !(s0 > -INFINITY) ? 0 : p.finished != nullptr && p.finished[row0 + beam] != 0 ? 2 : 1;
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
      start[beam] = s0;
      kind[beam] = what == 1 && !(m > -INFINITY) ? 0 : what;
      base[beam] = (double)m;
      log_sum[beam] = what == 1 && m > -INFINITY ? log(s) : 0.0;
    }
  }
  if (tid == 0) count = 0;
  __syncthreads();
  // larger scores first, then the lower place: (score, place) as words whose order is that; 0: no candidate
  uint64_t score[KPT], top = 0;
  uint32_t place[KPT], top_place = 0;
#pragma unroll
  for (int k = 0; k < KPT; k++) {
    const int c = tid + k * THREADS, beam = c / per;
    score[k] = 0;
    place[k] = 0;
    if (c < total) {
      if (kind[beam] == 1 && key[k] != 0) {
        score[k] = ordered((double)start[beam] + (((double)from_ordered((uint32_t)(key[k] >> 32)) - base[beam]) - log_sum[beam]));
        place[k] = ~((uint32_t)beam * (uint32_t)p.vocab + (0xFFFFFFFFu - (uint32_t)key[k]));
      } else if (kind[beam] == 2 && c == beam * per) {
        score[k] = ordered((double)start[beam] + 0.0);   // (the two zeros are one)
        place[k] = ~((uint32_t)beam * (uint32_t)p.vocab + (uint32_t)p.eos);
      }
      if (score[k] > top || (score[k] == top && place[k] > top_place)) {
        top = score[k];
        top_place = place[k];
      }
    }
  }
  const uint32_t words[3] = {(uint32_t)(top >> 32), (uint32_t)top, top_place};
  uint32_t low[3];
  wave_bound(words, n, low);
  if ((tid & 63) == 0)
    for (int k = 0; k < 3; k++) bounds[tid >> 6][k] = low[k];
  __syncthreads();
  uint64_t bound = 0;
  uint32_t bound_place = 0;
#pragma unroll
  for (int w = 0; w < WAVES; w++) {
    const uint64_t b = (uint64_t)bounds[w][0] << 32 | bounds[w][1];
    if (b > bound || (b == bound && bounds[w][2] > bound_place)) {
      bound = b;
      bound_place = bounds[w][2];
    }
  }
#pragma unroll
  for (int k = 0; k < KPT; k++)
    if (score[k] != 0 && (score[k] > bound || (score[k] == bound && place[k] >= bound_place))) {
      const int at = atomicAdd(&count, 1);
      found[at] = Scored{score[k], place[k]};
    }
  __syncthreads();
  const int have = count;
  auto write = [&](int slot, float value, int parent, int token, bool done) {
    p.out_scores[row0 + slot] = value;
    p.parent[row0 + slot] = parent;
    p.token[row0 + slot] = token;
    p.out_finished[row0 + slot] = done ? 1 : 0;
  };
  for (int c = tid / kRankLanes; c < have; c += THREADS / kRankLanes) {
    const Scored mine = found[c];
    const int rank = rank_of(have, [&](int k) { return found[k].score > mine.score || (found[k].score == mine.score && found[k].place > mine.place); });
    if (rank < n && tid % kRankLanes == 0) {
      const uint32_t place = ~mine.place;
      const int parent = (int)(place / (uint32_t)p.vocab), token = (int)(place % (uint32_t)p.vocab);
      write(rank, (float)from_ordered(mine.score), parent, token, kind[parent] == 2 || token == p.eos);
    }
  }
  for (int c = have + tid; c < n; c += THREADS) write(c, -INFINITY, c, p.eos >= 0 ? p.eos : 0, true);
}

// A thread handles the same 16 bytes of all beams of a batch row: it reads what moves, then writes it, so that the states
// change in place whatever the parents are.  Sources that several beams take come from the caches after the first read; a beam that
// is its own parent is not touched: its buffer descriptor is empty, which keeps the loads and stores free of branches and
// all of them in flight.  Bound by memory: 2 x 128 states of 2 MiB, 7 in 8 of them moving, 153 us (5.2 TB/s).
template <int MAX>
__global__ __launch_bounds__(kReorderThreads) void beam_reorder_kernel(BeamReorderParams p) {
  typedef __attribute__((ext_vector_type(4))) uint32_t u32x4;
  constexpr int64_t BYTES = kReorderThreads * 16;
  const int64_t at = (int64_t)blockIdx.x * BYTES;
  const uint32_t bytes = (uint32_t)min(p.row_bytes - at, BYTES);
  const int32_t* parent = p.parent + (int64_t)blockIdx.y * p.beams;
  char* base = static_cast<char*>(p.states[blockIdx.z]) + (int64_t)blockIdx.y * p.beams * p.row_bytes + at;
  const uint32_t off = threadIdx.x * 16;
  const int lane = threadIdx.x & 63;
  int parents = lane < p.beams ? parent[lane] : lane;
  u32x4 v[MAX];
  // beam j's 16 bytes; an empty descriptor where it does not move
  auto rows = [&](int j, bool source) {
    const int from = __builtin_amdgcn_readlane(parents, j);
    const bool moves = j < p.beams && from != j && from >= 0 && from < p.beams;
    return __builtin_amdgcn_make_buffer_rsrc(base + (moves ? (source ? from : j) : 0) * p.row_bytes, 0, moves ? (int)bytes : 0, 0x00027000);
  };
#pragma unroll
  for (int j = 0; j < MAX; j++) v[j] = __builtin_amdgcn_raw_buffer_load_b128(rows(j, true), (int)off, 0, 0);
  asm volatile("" : "+v"(parents));   // read out again below: 32 beams' worth overflow the scalar registers
#pragma unroll
  for (int j = 0; j < MAX; j++) __builtin_amdgcn_raw_buffer_store_b128(v[j], rows(j, false), (int)off, 0, 0);
}

// How the vocabulary is cut.  Pieces of 4096 logits, or 8192 where the rows alone fill the device; a workgroup works off several where their
// candidates would be more than the second launch's threads hold.
constexpr int kSmallPart = 4096, kLargePart = 8192, kMergeMost = 1024 * 8, kMergeMore = 512 * 4, kMergeFew = 256 * 4;
static_assert(kMaxBeams * kMaxBeams <= kMergeMost, "one piece a row at least");

struct Cut {
  int part, parts, chunks;
};
Cut cut(int64_t rows, int32_t beams, int32_t vocab, int units) {
  Cut c;
  c.part = vocab > kSmallPart && rows * ((vocab + kLargePart - 1) / kLargePart) >= 4 * units ? kLargePart : kSmallPart;
  const int all = (vocab + c.part - 1) / c.part, most = kMergeMost / (beams * beams);
  c.parts = (all + most - 1) / most;
  c.chunks = (all + c.parts - 1) / c.parts;
  return c;
}

template <typename T>
hipError_t select(BeamSelectParams p, const Cut& c, hipStream_t s) {
  constexpr int kSmall = kSmallPart / (kSelectThreads * Piece<T>::N), kLarge = kLargePart / (kSelectThreads * Piece<T>::N);
  const dim3 grid((unsigned)((int64_t)p.chunks * p.batch * p.beams));
  if (c.part == kSmallPart) hipLaunchKernelGGL((beam_chunk_kernel<T, kSmall>), grid, dim3(kSelectThreads), 0, s, p);
  else hipLaunchKernelGGL((beam_chunk_kernel<T, kLarge>), grid, dim3(kSelectThreads), 0, s, p);
  const hipError_t e = hipGetLastError();
  if (e != hipSuccess) return e;
  const int candidates = p.beams * p.beams * p.chunks;
  if (candidates <= kMergeFew) hipLaunchKernelGGL((beam_merge_kernel<256, 4>), dim3((unsigned)p.batch), dim3(256), 0, s, p);
  else if (candidates <= kMergeMore) hipLaunchKernelGGL((beam_merge_kernel<512, 4>), dim3((unsigned)p.batch), dim3(512), 0, s, p);
  else hipLaunchKernelGGL((beam_merge_kernel<1024, 8>), dim3((unsigned)p.batch), dim3(1024), 0, s, p);
  return hipGetLastError();
}

}  // namespace

int beam_select_chunks(int64_t rows, int32_t beams, int32_t vocab, int units) { return cut(rows, beams, vocab, units).chunks; }

hipError_t launch_beam_select(int dtype, BeamSelectParams p, int units, hipStream_t s) {
  const Cut c = cut((int64_t)p.batch * p.beams, p.beams, p.vocab, units);
  p.chunks = c.chunks;
  p.parts = c.parts;
  if (dtype == kBF16) return select<__bf16>(p, c, s);
  if (dtype == kF16) return select<_Float16>(p, c, s);
  return select<float>(p, c, s);
}

hipError_t launch_beam_reorder(const BeamReorderParams& p, int nstates, hipStream_t s) {
  const int64_t threads = p.row_bytes / 16;
  const dim3 grid((unsigned)((threads + kReorderThreads - 1) / kReorderThreads), (unsigned)p.batch, (unsigned)nstates);
  if (p.beams <= 4) hipLaunchKernelGGL(beam_reorder_kernel<4>, grid, dim3(kReorderThreads), 0, s, p);
  else if (p.beams <= 8) hipLaunchKernelGGL(beam_reorder_kernel<8>, grid, dim3(kReorderThreads), 0, s, p);
  else if (p.beams <= 16) hipLaunchKernelGGL(beam_reorder_kernel<16>, grid, dim3(kReorderThreads), 0, s, p);
  else hipLaunchKernelGGL(beam_reorder_kernel<32>, grid, dim3(kReorderThreads), 0, s, p);
  return hipGetLastError();
}

}  // namespace la2
