// The tiled matrix product (gfx950): one workgroup per TI x TJ tile of c (and piece of the reduction).
//
// Tiles of both operands stream from HBM straight into LDS (buffer loads with the LDS destination, 16 bytes per lane, no registers),
// one reduction step of 128 bytes a row (the 64 tile: two or three) ahead of the one being multiplied; a buffer descriptor of its own per step bounds them, so
// that rows behind a matrix' last one and elements behind the reduction's end arrive as 0.  One barrier per step.
//
// A wave owns (TI / WI) x (TJ / WJ) of the tile as 32 x 32 accumulators.  j is the accumulators' row index and i their column (a lane holds four
// consecutive j of one i), which makes the rows of c the contiguous direction.
//
// LDS layouts, in 16-byte chunks, unpadded because the direct loads write 1 KiB per wave instruction:
//   along   rows of 8 chunks (128 bytes of the reduction); chunk c of row i at c ^ (i / 2 % 8): the 16-byte reads of 16 lanes (16 rows, one
//           chunk) meet all 64 banks once
//   across  a row is one reduction index, T elements; 16-bit types: chunk c of row r at c ^ 4 (r % 4) (T = 64, two rows in 256 bytes: c ^ 4 (r / 2 % 2)): a
//           transposing read of 32 lanes (4 rows, 64 bytes of each) meets all banks once.  fp32: in place, lanes read consecutive elements.
//
// Bound by the matrix pipes and LDS together (a step of the 256 tile keeps each busy for 2048 cycles of about 3400 in the backward pass' launch).  16384 x 8192 x 2048 bf16: the
// weight's gradient 436 us (1.26 PFLOP/s), the input's 469, forward 490 and with gelu and kept sums 564; 8192 x 8192 x 8192 1.2 PFLOP/s.  fp32
// 4096 x 4096 x 4096: 142 TFLOP/s, the rate of the fp32 matrix instructions.
#ifndef LA2_LINEAR_TILES_H_
#define LA2_LINEAR_TILES_H_

#include "la2_bf16_common.h"
#include "la2_linear.h"

namespace la2 {
namespace linear {

using bf16k::f32x16;
using bf16k::i32x4;
using bf16k::lds_barrier;
using bf16k::lds_offset;
using bf16k::lds_read_tr;
using bf16k::s16x4;

// What one lane holds of 32 rows and one group of the reduction (16 elements of a 16-bit type, 8 of fp32): one 16-byte chunk.
template <typename E>
struct Frag {
  typedef typename Piece<E>::vec V;
  V v;
};
template <typename E>
__device__ __forceinline__ f32x16 multiply(const Frag<E>& a, const Frag<E>& b, f32x16 c) {
  return bf16k::mfma(a.v, b.v, c);
}
// fp32: the four elements of a lane's chunk in turn; lanes l and l + 32 hold the two reduction indices of an instruction, the same
// for both operands
template <>
__device__ __forceinline__ f32x16 multiply<float>(const Frag<float>& a, const Frag<float>& b, f32x16 c) {
#pragma unroll
  for (int e = 0; e < 4; e++) c = __builtin_amdgcn_mfma_f32_32x32x2f32(a.v[e], b.v[e], c, 0, 0, 0);
  return c;
}

// Direct load, 16 bytes per lane: LDS address lds + 16 lane, 0 for what lies outside the descriptor.  The compiler does not look into an asm
// statement for the wait states between a vector instruction that writes a scalar register (a readfirstlane of the descriptor) and a memory
// instruction that reads it, five; the statement brings them.
__device__ __forceinline__ void load_lds(i32x4 rsrc, uint32_t off, uint32_t lds) {
  asm volatile("s_mov_b32 m0, %2\n\ts_nop 4\n\tbuffer_load_dwordx4 %0, %1, 0 offen lds"
               :
               : "v"(off), "s"(rsrc), "s"(lds)
               : "m0", "memory");
}
constexpr uint32_t kOutside = 0x80000000u;   // behind every descriptor: tiles span less than 2 GiB (checked on the host)

constexpr int kStepBytes = 128;              // of the reduction, per row

template <int T>
__device__ __forceinline__ int across_swz(int row) {
  return T == 64 ? (row & 2) << 1 : (row & 3) << 2;   // T = 64: two rows in 256 bytes
}

// One operand's tile: T rows (i or j), a step of the reduction.
template <typename E, int T, bool ACROSS, int NW>
struct Operand {
  static constexpr int KE = kStepBytes / (int)sizeof(E);   // reduction elements of a step
  static constexpr int BYTES = T * kStepBytes;
  static constexpr int LOADS = BYTES / 1024 / NW;          // wave instructions per wave
  static constexpr int ROW = ACROSS ? T * (int)sizeof(E) : kStepBytes;
  static_assert(LOADS >= 1 && LOADS * NW * 1024 == BYTES, "whole instructions per wave");
  uint32_t off[LOADS];
  int first[LOADS];        // along: the reduction element that the lane's chunk starts with
  const char* base;        // this tile's start in the step at hand
  int64_t step;            // bytes between steps
  int64_t left;            // bytes from base to the end of the tile's last row (along) or of its columns in the last row (across)
  int64_t most;            // across: what a step's rows span
  int wave;

  __device__ __forceinline__ static int swz(int row) {
    if (!ACROSS) return (row >> 1) & 7;
    return sizeof(E) == 2 ? across_swz<T>(row) : 0;
  }
  // rows row0 .. of `rows`, the reduction's elements r0 .. r1 - 1
  __device__ __forceinline__ void start(const void* p, int64_t ld, int64_t row0, int64_t rows, int64_t r0, int64_t r1, int w, int lane) {
    constexpr int S = (int)sizeof(E);
    wave = w;
#pragma unroll
    for (int k = 0; k < LOADS; k++) {
      const int byte = (w * LOADS + k) * 1024 + lane * 16;
      const int row = byte / ROW, chunk = (byte % ROW / 16) ^ swz(row);
      off[k] = (uint32_t)(row * ld * S + chunk * 16);
      first[k] = chunk * (16 / S);
    }
    // to whole chunks: a chunk that is partly behind the end would be 0 altogether (its rest is there: rows are whole chunks, see
    // la2_linear.hip)
    constexpr int64_t C = 16 / S;
    if (ACROSS) {
      const int64_t have = min((rows - row0 + C - 1) / C * C, (int64_t)T);
      base = static_cast<const char*>(p) + (r0 * ld + row0) * S;
      step = (int64_t)KE * ld * S;
      left = ((r1 - r0 - 1) * ld + have) * S;
      most = ((KE - 1) * ld + have) * S;
    } else {
      const int64_t have = min(rows - row0, (int64_t)T);
      base = static_cast<const char*>(p) + (row0 * ld + r0) * S;
      step = kStepBytes;
      left = ((have - 1) * ld + (r1 - r0 + C - 1) / C * C) * S;
      most = left;
    }
  }
  // The loads of the step at hand, k of LOADS; `rem`: what is left of the reduction in it, in elements
  __device__ __forceinline__ void load(int k, uint32_t lds, int rem) const {
    const uint64_t at = (uint64_t)base;
    const int64_t bytes = left < most ? left : most;
    i32x4 rsrc;
    rsrc[0] = (int)(uint32_t)at;
    rsrc[1] = (int)(uint32_t)(at >> 32);
    rsrc[2] = (int)(uint32_t)bytes;
    rsrc[3] = 0x00027000;
#pragma unroll
    for (int e = 0; e < 3; e++) rsrc[e] = __builtin_amdgcn_readfirstlane(rsrc[e]);
    const uint32_t o = ACROSS || first[k] < rem ? off[k] : kOutside;
    load_lds(rsrc, o, __builtin_amdgcn_readfirstlane((int)(lds + (uint32_t)(wave * LOADS + k) * 1024u)));
  }
  __device__ __forceinline__ void advance() {
    base += step;
    left -= step;
  }
};

// Rows t * 32 .. + 31 (t counted in the tile) of group g of the step
template <typename E, int T, bool ACROSS>
__device__ __forceinline__ Frag<E> read(const char* tile, int t, int g, int lane) {
  const int l32 = lane & 31, hh = lane >> 5;
  Frag<E> f;
  if constexpr (!ACROSS) {
    const int row = t * 32 + l32;
    f.v = *reinterpret_cast<const typename Piece<E>::vec*>(tile + row * kStepBytes + (((2 * g + hh) ^ ((row >> 1) & 7)) << 4));
  } else if constexpr (sizeof(E) == 2) {
    // lane s of 16 passes row r + s / 4, elements 4 (s % 4) .. + 3 of its 16 columns, and gets its own column of the 4 rows
    const int s = lane & 15, half = (lane >> 4) & 1;
    const int r = 16 * g + 8 * hh + (s >> 2);
    const int chunk = 4 * t + 2 * half + ((s & 3) >> 1);
    union { struct { s16x4 lo, hi; } h; typename Piece<E>::vec v; } u;
    const int place = ((chunk ^ across_swz<T>(r)) << 4) + 8 * (s & 1);   // of row r + 4 as well
    u.h.lo = lds_read_tr(tile + r * (2 * T) + place);
    u.h.hi = lds_read_tr(tile + (r + 4) * (2 * T) + place);
    f.v = u.v;
  } else {
#pragma unroll
    for (int e = 0; e < 4; e++) f.v[e] = reinterpret_cast<const float*>(tile)[(8 * g + 4 * hh + e) * T + t * 32 + l32];
  }
  return f;
}

// Workgroups on neighbouring tiles share an XCD (they are dealt out to the eight in turn), in bands of kBand tile rows, so that an
// XCD's L2 holds the rows and columns that its tiles have in common.
constexpr int kXcds = 8, kBand = 4;
__device__ __forceinline__ void place(uint32_t wg, uint32_t tiles_i, uint32_t tiles_j, uint32_t& ti, uint32_t& tj) {
  const uint32_t total = tiles_i * tiles_j, whole = total / kXcds * kXcds;
  if (wg < whole) wg = (wg % kXcds) * (whole / kXcds) + wg / kXcds;
  const uint32_t band = wg / (kBand * tiles_j), first = band * kBand;
  const uint32_t height = min((uint32_t)kBand, tiles_i - first), in = wg - first * tiles_j;
  ti = first + in % height;
  tj = in / height;
}

template <int N>
__device__ __forceinline__ void wait_loads() {   // until at most N of this wave's loads are on their way
  asm volatile("s_waitcnt vmcnt(%0)" ::"n"(N) : "memory");
}

// A tile's shape: TI x TJ, WI x WJ waves, STAGES buffers
template <int TI_, int TJ_, int WI_, int WJ_, int STAGES_>
struct Shape {
  static constexpr int TI = TI_, TJ = TJ_, WI = WI_, WJ = WJ_, STAGES = STAGES_, NW = WI * WJ, THREADS = 64 * NW;
  static constexpr int BYTES = (TI + TJ) * kStepBytes * STAGES;
  static_assert(TI == TJ && THREADS == kTileThreads[TI / 128], "as planned");
};

// Workgroup `wg` of the tiles of p
template <typename E, typename S, bool AA, bool AB>
__device__ __forceinline__ void product(const ProductParams& p, uint32_t wg, char* lds) {
  constexpr int TI = S::TI, TJ = S::TJ, WJ = S::WJ, NW = S::NW, NI = TI / S::WI / 32, NJ = TJ / WJ / 32, STAGES = S::STAGES;
  constexpr int KE = kStepBytes / (int)sizeof(E), GROUPS = kStepBytes / 32;
  using A = Operand<E, TI, AA, NW>;
  using B = Operand<E, TJ, AB, NW>;
  constexpr int STAGE = A::BYTES + B::BYTES, LOADS = A::LOADS + B::LOADS;
  constexpr int ROWF = 32 * NJ + 4;   // floats of a row in the epilogue's staging
  static_assert(NW * 32 * ROWF * 4 <= S::BYTES && STAGE * STAGES == S::BYTES, "the staging fits");
  const int lane = threadIdx.x & 63;
  const int w = __builtin_amdgcn_readfirstlane((int)(threadIdx.x >> 6)), wi = w / WJ, wj = w % WJ;
  uint32_t ti, tj;
  const uint32_t tiles_i = (uint32_t)((p.I + TI - 1) / TI), tiles_j = (uint32_t)((p.J + TJ - 1) / TJ);
  const uint32_t split = wg / (tiles_i * tiles_j);
  place(wg % (tiles_i * tiles_j), tiles_i, tiles_j, ti, tj);
  const int64_t i0 = (int64_t)ti * TI, j0 = (int64_t)tj * TJ, r0 = split * p.span, r1 = min(p.R, r0 + p.span);

  f32x16 acc[NI][NJ];
#pragma unroll
  for (int i = 0; i < NI; i++)
#pragma unroll
    for (int j = 0; j < NJ; j++) acc[i][j] = bf16k::zero16();

  A a;
  B b;
  a.start(p.a, p.lda, i0, p.I, r0, r1, w, lane);
  b.start(p.b, p.ldb, j0, p.J, r0, r1, w, lane);
  const uint32_t at = lds_offset(lds);
  int rem = (int)(r1 - r0);   // of the reduction, from the next step to be loaded on
  const int steps = (rem + KE - 1) / KE;
  auto load = [&](int stage) {
#pragma unroll
    for (int k = 0; k < A::LOADS; k++) a.load(k, at + stage * STAGE, rem);
#pragma unroll
    for (int k = 0; k < B::LOADS; k++) b.load(k, at + stage * STAGE + A::BYTES, rem);
    a.advance();
    b.advance();
    rem -= KE;
  };
#pragma unroll
  for (int s = 0; s < STAGES - 1; s++)
    if (s < steps) load(s);
  int here = 0, next = STAGES - 1;
  for (int t = 0; t < steps; t++) {
    if (t + STAGES - 1 <= steps) wait_loads<(STAGES - 2) * LOADS>();   // this step's have arrived: those of STAGES - 2 behind it are under way
    else wait_loads<0>();
    lds_barrier();   // everybody's have, and nobody reads the buffer of the step before any more
    if (t + STAGES - 1 < steps) load(next);
    const char* tile = lds + here * STAGE;
    // A group's operands are read while the group before it is multiplied, in that order of issue: left to itself the compiler reads
    // right in front of the products (16384 x 8192 x 2048, the weight's gradient: 453 us so, 436 in this order)
    Frag<E> fa[2][NI], fb[2][NJ];
    auto fetch = [&](int g) {
#pragma unroll
      for (int j = 0; j < NJ; j++) fb[g & 1][j] = read<E, TJ, AB>(tile + A::BYTES, wj * NJ + j, g, lane);
#pragma unroll
      for (int i = 0; i < NI; i++) fa[g & 1][i] = read<E, TI, AA>(tile, wi * NI + i, g, lane);
    };
    constexpr int READS = NI * (AA ? 2 : 1) + NJ * (AB ? 2 : 1);   // instructions of a 16-bit group
    fetch(0);
#pragma unroll
    for (int g = 0; g < GROUPS; g++) {
      if (g + 1 < GROUPS) fetch(g + 1);
#pragma unroll
      for (int i = 0; i < NI; i++)
#pragma unroll
        for (int j = 0; j < NJ; j++) acc[i][j] = multiply<E>(fb[g & 1][j], fa[g & 1][i], acc[i][j]);
      if (sizeof(E) == 2) {
        constexpr int kLdsReads = 0x100, kProducts = 0x8;
        if (g == 0) __builtin_amdgcn_sched_group_barrier(kLdsReads, READS, 0);
        if (g + 1 < GROUPS) __builtin_amdgcn_sched_group_barrier(kLdsReads, READS, 0);
        __builtin_amdgcn_sched_group_barrier(kProducts, NI * NJ, 0);
      }
    }
    here = here + 1 == STAGES ? 0 : here + 1;
    next = next + 1 == STAGES ? 0 : next + 1;
  }
  lds_barrier();   // the tiles are done with: each wave stages its rows in its own part of them

  constexpr int N = Piece<E>::N, LPR = 32 * NJ / N, RPI = 64 / LPR;   // lanes of a row, rows of an instruction
  float* stage = reinterpret_cast<float*>(lds) + w * 32 * ROWF;
  const int l32 = lane & 31, hh = lane >> 5;
  const int row0 = lane / LPR, col = lane % LPR * N;
  const int64_t cj = j0 + wj * NJ * 32 + col;
  float bias[N];
  load_floats(p.splits == 1 ? p.bias : nullptr, cj, p.J, 0.f, bias);
  with_act(p.act, [&](auto act) {
#pragma unroll
    for (int i = 0; i < NI; i++) {
#pragma unroll
      for (int j = 0; j < NJ; j++)
#pragma unroll
        for (int q = 0; q < 4; q++) {
          const bf16k::f32x4 four = {acc[i][j][4 * q], acc[i][j][4 * q + 1], acc[i][j][4 * q + 2], acc[i][j][4 * q + 3]};
          *reinterpret_cast<bf16k::f32x4*>(stage + l32 * ROWF + 32 * j + 8 * q + 4 * hh) = four;
        }
      if (cj >= p.J) continue;
#pragma unroll
      for (int k = 0; k < 32 / RPI; k++) {
        const int row = k * RPI + row0;
        const int64_t ci = i0 + (wi * NI + i) * 32 + row;
        if (ci >= p.I) continue;
        float v[N];
#pragma unroll
        for (int e = 0; e < N; e += 4) {
          const bf16k::f32x4 four = *reinterpret_cast<const bf16k::f32x4*>(stage + row * ROWF + col + e);
#pragma unroll
          for (int f = 0; f < 4; f++) v[e + f] = four[f];
        }
        if (p.splits == 1) finish<E, decltype(act)::value, N>(p, ci, cj, bias, v);
        else store_floats(p.partial + (split * p.I + ci) * p.J, cj, p.J, v);
      }
    }
  });
}

template <typename E, typename S>
__global__ __launch_bounds__(S::THREADS) void product_kernel(ProductParams p) {
  __shared__ __align__(1024) char lds[S::BYTES];
  product<E, S, false, false>(p, blockIdx.x, lds);
}

template <typename E, typename S>
__global__ __launch_bounds__(S::THREADS) void product_pair_kernel(PairParams q) {
  __shared__ __align__(1024) char lds[S::BYTES];
  uint32_t wg = blockIdx.x;
  const uint32_t products = (uint32_t)(q.groups[0] + q.groups[1]), first = (uint32_t)(q.weight_first ? q.groups[1] : q.groups[0]);
  if (wg < products) {
    const bool weight = (wg < first) == (q.weight_first != 0);
    if (wg >= first) wg -= first;
    if (weight) product<E, S, true, true>(q.p[1], wg, lds);
    else product<E, S, false, true>(q.p[0], wg, lds);
    return;
  }
  // 16 columns of the sums, in a fixed order
  constexpr int SLICES = S::THREADS / 16;
  float* part = reinterpret_cast<float*>(lds);
  const int col = threadIdx.x % 16, slice = threadIdx.x / 16;
  const int64_t j = (int64_t)(wg - products) * 16 + col;
  float v = 0.f;
  if (j < q.width) {
#pragma unroll 8
    for (int r = slice; r < q.count; r += SLICES) v += q.partial[(int64_t)r * q.width + j];
  }
  part[slice * 17 + col] = v;
  __syncthreads();
  if (slice != 0 || j >= q.width) return;
  v = 0.f;
#pragma unroll
  for (int i = 0; i < SLICES; i++) v += part[i * 17 + col];
  q.sums[j] = v;
}

// The tiles.  Two buffers of the large one take 128 of a unit's 160 KiB of LDS, so that it has a unit for itself; the small ones, whose steps are shorter than a load takes, load further ahead.
using Tile64 = Shape<64, 64, 2, 2, 4>;        // two workgroups on a unit
using Tile64Dense = Shape<64, 64, 2, 2, 3>;   // three, where there are more than two for each (1001 x 1111 x 999 fp16 backward: 28.2 us with four buffers, 26.7 so)
using Tile128 = Shape<128, 128, 2, 2, 2>;
using Tile256 = Shape<256, 256, 2, 4, 2>;

template <typename E, typename S>
hipError_t launch_one(const ProductParams& p, hipStream_t s) {
  const int64_t tiles = ((p.I + S::TI - 1) / S::TI) * ((p.J + S::TJ - 1) / S::TJ);
  hipLaunchKernelGGL((product_kernel<E, S>), dim3((unsigned)(tiles * p.splits)), dim3(S::THREADS), 0, s, p);
  return hipGetLastError();
}
template <typename E, typename S>
hipError_t launch_both(PairParams q, hipStream_t s) {
  int64_t groups = 0;
  for (int k = 0; k < 2; k++) {
    const ProductParams& p = q.p[k];
    if (q.groups[k] != 0) q.groups[k] = (int32_t)(((p.I + S::TI - 1) / S::TI) * ((p.J + S::TJ - 1) / S::TJ) * p.splits);
    groups += q.groups[k];
  }
  q.weight_first = q.p[1].span > q.p[0].span;
  if (q.partial != nullptr) groups += (q.width + 15) / 16;
  hipLaunchKernelGGL((product_pair_kernel<E, S>), dim3((unsigned)groups), dim3(S::THREADS), 0, s, q);
  return hipGetLastError();
}

template <typename E>
hipError_t launch_product(int tile, const ProductParams& p, hipStream_t s) {
  if (tile == kTile256) return launch_one<E, Tile256>(p, s);
  if (tile == kTile128) return launch_one<E, Tile128>(p, s);
  const int64_t groups = ((p.I + 63) / 64) * ((p.J + 63) / 64) * p.splits;
  return groups > 2 * (int64_t)device_units() ? launch_one<E, Tile64Dense>(p, s) : launch_one<E, Tile64>(p, s);
}
template <typename E>
hipError_t launch_pair(int tile, const PairParams& p, hipStream_t s) {
  if (tile == kTile256) return launch_both<E, Tile256>(p, s);
  if (tile == kTile128) return launch_both<E, Tile128>(p, s);
  int64_t groups = 0;
  for (int k = 0; k < 2; k++)
    if (p.groups[k] != 0) groups += ((p.p[k].I + 63) / 64) * ((p.p[k].J + 63) / 64) * p.p[k].splits;
  return groups > 2 * (int64_t)device_units() ? launch_both<E, Tile64Dense>(p, s) : launch_both<E, Tile64>(p, s);
}

}  // namespace linear
}  // namespace la2
#endif
