// Low-rank adapters of many requests beside a shared projection, and their
// gradients. With h = A[id] x of rank r, Y = fp16(base + s[id] B[id] h): two
// skinny products through r numbers per token.
//
//   shrink_kernel  h, as partial sums over ranges of the width. Both operands
//                  are contiguous along the contraction, so that a lane's
//                  16-byte loads are MFMA operands as they come: no LDS.
//   expand_kernel  adds the ranges, multiplies with the other factor and adds
//                  to the base. The contraction runs across the factor's rows,
//                  so the factor goes through LDS and transposing reads.
//   outer_kernel   an adapter's sums over its tokens of h times input (the
//                  factors' gradients), split over the tokens where the grid
//                  is small; outer_reduce_kernel adds the splits in order.
//   sort_kernel    tokens in the order of their adapters, and tiles of 32 of
//                  them, so that an MFMA's tokens share a factor.
//
// Both factors are kept rank by rank ([adapter][rank][width]): the backward
// pass is the forward one with the factors exchanged (u = B^T dY by
// shrink_kernel, s A^T u by expand_kernel).
//
// h and u are fp32. Where they are operands of fp16 MFMAs they are scaled by a
// power of two, so that the largest lies in [2^13, 2^14), and split into the
// nearest fp16 and the rest's nearest fp16: 22 bits or, for small ones, 2^-38
// of the largest. Two MFMAs instead of one; the launches are bound by memory.

#include <hip/hip_fp16.h>
#include <hip/hip_runtime.h>

#include <algorithm>
#include <cstring>

#include "internal.h"
#include "lanes.h"
#include "lowrank.h"

namespace {

using namespace spdp_low;

using namespace spdp_dev;

typedef float float4v __attribute__((ext_vector_type(4)));

constexpr int kTile = 32;  // tokens of a tile
constexpr int kThreads = 256;
constexpr int kWaves = 4;

// The tokens of tile `block` to tok[0 .. kTile - 1] (places past the count
// repeat one of them); false: no tile. Every wave does it alike.
__device__ __forceinline__ bool take_tile(const Tokens& t, int block, int* tok, int& adapter, int& count) {
  const int lane = threadIdx.x & 63;
  if (t.ids == nullptr) {
    adapter = 0;
    count = min(kTile, t.n_tokens - block * kTile);
    if (lane < kTile) tok[lane] = block * kTile + min(lane, count - 1);
  } else if (t.tiles == nullptr) {
    // the tile of token `block`, which has to be the first, 33rd, ... of its adapter
    int id = lane < t.n_tokens ? t.ids[lane] : -2;
    if (id >= t.count || (lane < t.n_tokens && id < 0)) id = -1;
    adapter = __builtin_amdgcn_readlane(id, block);
    const uint64_t same = __ballot(lane < t.n_tokens && id == adapter);
    const int first = __popcll(same & ((1ull << block) - 1));
    if (first % kTile != 0) return false;
    count = min(kTile, (int)__popcll(same) - first);
    const int rank = (int)__popcll(same & ((1ull << lane) - 1)) - first;
    if ((same >> lane & 1) && rank >= 0 && rank < kTile) tok[rank] = lane;
    if (lane >= count && lane < kTile) tok[lane] = block;
  } else {
    const Tile d = t.tiles[block];
    adapter = d.adapter;
    count = d.count;
    if (count == 0) return false;
    if (lane < kTile) tok[lane] = t.perm[d.start + min(lane, count - 1)];
  }
  wave_fence();
  return true;
}

// ---------------------------------------------------------------------------
// Shrink. A workgroup owns a tile of tokens and a range of the width, its four
// waves every fourth step of 32 columns; 16x16x32 MFMAs with the tokens as
// rows. The waves' sums are added in LDS.

constexpr int kStep = 32;

template <int RB>  // 16 RB ranks
__global__ __launch_bounds__(kThreads) void shrink_kernel(ShrinkArgs a) {
  __shared__ int tok[kTile];
  extern __shared__ __attribute__((aligned(16))) float red[];  // [wave][token][16 RB]
  const Shrink& m = a.m[blockIdx.z];
  const int lane = threadIdx.x & 63;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  int adapter, count;
  if (!take_tile(a.t, blockIdx.x, tok, adapter, count) || adapter < 0) return;
  const int steps = (m.width + kStep - 1) / kStep;
  const int s0 = (int)blockIdx.y * m.per, s1 = min(steps, s0 + m.per);
  if (s0 >= steps) return;  // the grid has the most ranges of the launch's products
  const int k0 = 8 * (lane >> 4);
  const uint16_t *px[2], *pf[RB];
#pragma unroll
  for (int i = 0; i < 2; ++i) px[i] = m.in + (size_t)tok[16 * i + (lane & 15)] * m.width + k0;
#pragma unroll
  for (int j = 0; j < RB; ++j)
    pf[j] = m.factor + ((size_t)adapter * a.rank + min(16 * j + (lane & 15), a.rank - 1)) * m.width + k0;

  float4v acc[2][RB];
#pragma unroll
  for (int i = 0; i < 2; ++i)
#pragma unroll
    for (int j = 0; j < RB; ++j) acc[i][j] = float4v{0, 0, 0, 0};
  const bool two = count > 16;
  // steps whose columns all lie inside the width, kDeep of them at a time
  constexpr int kDeep = RB == 8 ? 2 : 4;
  const int whole = min(s1, m.width / kStep);
  int s = s0 + wave;
  auto multiply = [&](const half8 (&x)[2], const half8 (&f)[RB]) __attribute__((always_inline)) {
#pragma unroll
    for (int j = 0; j < RB; ++j) {
      acc[0][j] = __builtin_amdgcn_mfma_f32_16x16x32_f16(x[0], f[j], acc[0][j], 0, 0, 0);
      if (two) acc[1][j] = __builtin_amdgcn_mfma_f32_16x16x32_f16(x[1], f[j], acc[1][j], 0, 0, 0);
    }
  };
  for (; s + (kDeep - 1) * kWaves < whole; s += kDeep * kWaves) {
    half8 x[kDeep][2], f[kDeep][RB];
#pragma unroll
    for (int d = 0; d < kDeep; ++d) {
      const int at = (s + d * kWaves) * kStep;
      x[d][0] = load8(px[0] + at);
      x[d][1] = two ? load8(px[1] + at) : x[d][0];
#pragma unroll
      for (int j = 0; j < RB; ++j) f[d][j] = load8(pf[j] + at);
    }
#pragma unroll
    for (int d = 0; d < kDeep; ++d) multiply(x[d], f[d]);
  }
  for (; s < s1; s += kWaves) {
    const int at = s * kStep;
    const int left = m.width - at - k0;
    half8 x[2], f[RB];
#pragma unroll
    for (int i = 0; i < 2; ++i) x[i] = load8_inside(px[i] + at, left);
#pragma unroll
    for (int j = 0; j < RB; ++j) f[j] = load8_inside(pf[j] + at, left);
    multiply(x, f);
  }

  // register e of block (i, j): token 16 i + 4 (lane / 16) + e, rank 16 j + lane mod 16
#pragma unroll
  for (int i = 0; i < 2; ++i)
#pragma unroll
    for (int j = 0; j < RB; ++j)
#pragma unroll
      for (int e = 0; e < 4; ++e)
        red[((wave * kTile + 16 * i + 4 * (lane >> 4) + e) * RB + j) * 16 + (lane & 15)] = acc[i][j][e];
  __syncthreads();
  float* const part = m.part + (size_t)blockIdx.y * a.t.n_tokens * a.rank;
  for (int q = threadIdx.x; q < count * 16 * RB; q += kThreads) {
    const int t = q / (16 * RB), j = q % (16 * RB);
    if (j >= a.rank) continue;
    float sum = red[q];
#pragma unroll
    for (int w = 1; w < kWaves; ++w) sum += red[w * kTile * 16 * RB + q];
    part[(size_t)tok[t] * a.rank + j] = sum;
  }
}

// ---------------------------------------------------------------------------
// Power-of-two scales and the split into two fp16.

// 2^e with 2^e largest in [2^13, 2^14), and 2^-e
__device__ __forceinline__ void pick_scale(float largest, float& up, float& down) {
  const int e = max((int)(__float_as_uint(largest) >> 23), 14);
  up = __uint_as_float((uint32_t)(267 - e) << 23);
  down = __uint_as_float((uint32_t)(e - 13) << 23);
}
__device__ __forceinline__ float finite_abs(float v) {
  const float a = fabsf(v);
  return a < __builtin_inff() ? a : 0.0f;
}
__device__ __forceinline__ void split2(float v, _Float16& hi, _Float16& lo) {
  hi = (_Float16)v;
  const float rest = v - (float)hi;
  lo = fabsf(v) < __builtin_inff() ? (_Float16)rest : (_Float16)0;
}

// ---------------------------------------------------------------------------
// Expand. A workgroup owns a tile of tokens and `blocks` blocks of 256
// columns, each wave 64 columns of a block. The factor's 64 columns go through
// the wave's own LDS into the MFMA's B operand, the sums back through it, so
// that base and output are read and written 128 bytes of a token at a time.

constexpr int kCols = 64;        // columns of a wave
constexpr int kBlock = kCols * kWaves;
constexpr int kFactorRow = 144;  // bytes of a factor row in LDS: 64 fp16 + 16, which spreads the rows over the banks
constexpr int kOutRow = 72;      // floats of a row of sums

template <int RB>
struct ExpandCfg {
  static constexpr int kRank = 16 * RB;
  static constexpr int kActRow = 2 * kRank + 16;  // bytes
  static constexpr int kWave = kRank * kFactorRow > 4 * kTile * kOutRow ? kRank * kFactorRow : 4 * kTile * kOutRow;
  static constexpr int kLds = 2 * kTile * kActRow + kWaves * kWave;
};

template <int RB>
__global__ __launch_bounds__(kThreads) void expand_kernel(ExpandArgs a) {
  using C = ExpandCfg<RB>;
  __shared__ int tok[kTile];
  __shared__ float mult[kTile];
  extern __shared__ __attribute__((aligned(16))) unsigned char lds[];
  const Expand& m = a.m[blockIdx.z];
  const int lane = threadIdx.x & 63;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  if ((int)blockIdx.x * a.blocks * kBlock >= m.width) return;
  int adapter, count;
  if (!take_tile(a.t, blockIdx.y, tok, adapter, count)) return;
  unsigned char* const act_hi = lds;
  unsigned char* const act_lo = lds + kTile * C::kActRow;
  unsigned char* const mine = lds + 2 * kTile * C::kActRow + wave * C::kWave;

  if (adapter >= 0) {
    // eight threads a token
    const int t = threadIdx.x >> 3;
    const size_t row = (size_t)tok[t] * a.rank;
    const size_t plane = (size_t)a.t.n_tokens * a.rank;
    float v[2 * RB];
    float largest = 0.0f;
#pragma unroll
    for (int i = 0; i < 2 * RB; ++i) {
      const int j = 8 * i + (threadIdx.x & 7);
      v[i] = 0.0f;
      if (j < a.rank)
        for (int s = 0; s < m.splits; ++s) v[i] += m.part[s * plane + row + j];
      if (m.keep != nullptr && blockIdx.x == 0 && t < count && j < a.rank) m.keep[row + j] = v[i];
      largest = fmaxf(largest, finite_abs(v[i]));
    }
#pragma unroll
    for (int d = 1; d < 8; d <<= 1) largest = fmaxf(largest, __shfl_xor(largest, d));
    float up, down;
    pick_scale(largest, up, down);
#pragma unroll
    for (int i = 0; i < 2 * RB; ++i) {
      _Float16 hi, lo;
      split2(v[i] * up, hi, lo);
      const int at = t * C::kActRow + 2 * (8 * i + (threadIdx.x & 7));
      *reinterpret_cast<_Float16*>(act_hi + at) = hi;
      *reinterpret_cast<_Float16*>(act_lo + at) = lo;
    }
    if ((threadIdx.x & 7) == 0) mult[t] = down * m.scale[adapter];
  } else if (m.keep != nullptr && blockIdx.x == 0) {
    for (int q = threadIdx.x; q < count * a.rank; q += kThreads)
      m.keep[(size_t)tok[q / a.rank] * a.rank + q % a.rank] = 0.0f;
  }
  __syncthreads();

  for (int b = 0; b < a.blocks; ++b) {
    const int n0 = ((int)blockIdx.x * a.blocks + b) * kBlock + wave * kCols;
    if (n0 >= m.width) return;
    const int col = n0 + 8 * (lane & 7);
    const int left = m.width - col;  // columns of the lane's eight that there are; may be negative
    half8 base[4];
#pragma unroll
    for (int p = 0; p < 4; ++p) {
      const int t = 8 * p + (lane >> 3);
      if (t < count && left > 0) base[p] = load8_inside(m.base + (size_t)tok[t] * m.width + col, left);
    }
    if (adapter >= 0) {
      const uint16_t* const f = m.factor + (size_t)adapter * a.rank * m.width + col;
#pragma unroll
      for (int p = 0; p < 2 * RB; ++p) {
        const int j = 8 * p + (lane >> 3);
        half8 v = half8{0, 0, 0, 0, 0, 0, 0, 0};
        if (j < a.rank && left > 0) v = load8_inside(f + (size_t)j * m.width, left);
        *reinterpret_cast<half8*>(mine + j * kFactorRow + 16 * (lane & 7)) = v;
      }
      wave_fence();
      float16v acc[2] = {float16v{}, float16v{}};
#pragma unroll
      for (int k = 0; k < RB; ++k) {
        const int at = (lane & 31) * C::kActRow + 2 * (16 * k + 8 * (lane >> 5));
        const half8 hi = *reinterpret_cast<const half8*>(act_hi + at), lo = *reinterpret_cast<const half8*>(act_lo + at);
#pragma unroll
        for (int i = 0; i < 2; ++i) {
          const half8 v = read_transposed(mine, kFactorRow, 16 * k, 32 * i);
          acc[i] = __builtin_amdgcn_mfma_f32_32x32x16_f16(hi, v, acc[i], 0, 0, 0);
          acc[i] = __builtin_amdgcn_mfma_f32_32x32x16_f16(lo, v, acc[i], 0, 0, 0);
        }
      }
      wave_fence();
      // register e: token 8 (e / 4) + 4 (lane / 32) + e mod 4, column lane mod 32
      float* const sums = reinterpret_cast<float*>(mine);
#pragma unroll
      for (int i = 0; i < 2; ++i)
#pragma unroll
        for (int e = 0; e < 16; ++e)
          sums[(8 * (e >> 2) + 4 * (lane >> 5) + (e & 3)) * kOutRow + 32 * i + (lane & 31)] = acc[i][e];
      wave_fence();
    }
#pragma unroll
    for (int p = 0; p < 4; ++p) {
      const int t = 8 * p + (lane >> 3);
      if (t >= count || left <= 0) continue;
      half8 y = base[p];
      if (adapter >= 0) {
        const float* const sums = reinterpret_cast<const float*>(mine) + t * kOutRow + 8 * (lane & 7);
        const float by = mult[t];
#pragma unroll
        for (int e = 0; e < 8; ++e) y[e] = (_Float16)__fmaf_rn(by, sums[e], (float)base[p][e]);
      }
      store8_inside(m.out + (size_t)tok[t] * m.width + col, y, left);
    }
    wave_fence();
  }
}

// ---------------------------------------------------------------------------
// Outer: for an adapter, out[j][f] = scale * sum over its tokens of act[t][j]
// in[t][f]. A workgroup owns 64 columns, all ranks and a range of the tokens,
// each wave every fourth group of 16 tokens (an MFMA's k); the input goes
// through the wave's LDS and transposing reads, and the waves' sums are added
// in LDS at the end.

constexpr int kGroup = 16;  // tokens of an MFMA

template <int RB>  // 32 RB ranks
__global__ __launch_bounds__(kThreads) void outer_kernel(OuterArgs a) {
  constexpr int kRed = 4 * kWaves * 2 * 16 * 64;
  constexpr int kIn = kWaves * kGroup * kFactorRow;
  __shared__ __attribute__((aligned(16))) unsigned char lds[kRed > kIn ? kRed : kIn];
  __shared__ float most[kWaves];
  const int lane = threadIdx.x & 63;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int which = (int)blockIdx.z / a.count, adapter = (int)blockIdx.z % a.count;
  const Outer& m = a.m[which];
  const int f0 = (int)blockIdx.x * kCols;
  if (f0 >= m.width) return;
  int t0 = a.first ? a.first[adapter] : 0;
  int t1 = a.first ? a.first[adapter + 1] : adapter == 0 ? a.n_tokens : 0;
  const int per = ((t1 - t0 + a.splits - 1) / a.splits + kGroup - 1) / kGroup * kGroup;
  t0 = min(t1, t0 + (int)blockIdx.y * per);
  t1 = min(t1, t0 + per);

  float largest = 0.0f;
  for (int q = threadIdx.x; q < (t1 - t0) * a.rank; q += kThreads) {
    const int p = t0 + q / a.rank;
    const int t = a.perm ? a.perm[p] : p;
    largest = fmaxf(largest, finite_abs(m.act[(size_t)t * a.rank + q % a.rank]));
  }
#pragma unroll
  for (int d = 1; d < 64; d <<= 1) largest = fmaxf(largest, __shfl_xor(largest, d));
  if (lane == 0) most[wave] = largest;
  __syncthreads();
#pragma unroll
  for (int w = 0; w < kWaves; ++w) largest = fmaxf(largest, most[w]);
  float up, down;
  pick_scale(largest, up, down);

  float16v acc[RB][2];
#pragma unroll
  for (int j = 0; j < RB; ++j) acc[j][0] = acc[j][1] = float16v{};
  unsigned char* const mine = lds + wave * kGroup * kFactorRow;
  const int col = f0 + 8 * (lane & 7);
  const int left = m.width - col;
  for (int g = t0 + wave * kGroup; g < t1; g += kWaves * kGroup) {
#pragma unroll
    for (int p = 0; p < 2; ++p) {
      const int at = g + 8 * p + (lane >> 3);
      half8 v = half8{0, 0, 0, 0, 0, 0, 0, 0};
      if (at < t1 && left > 0) v = load8_inside(m.in + (size_t)(a.perm ? a.perm[at] : at) * m.width + col, left);
      *reinterpret_cast<half8*>(mine + (8 * p + (lane >> 3)) * kFactorRow + 16 * (lane & 7)) = v;
    }
    half8 hi[RB], lo[RB];
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      const int at = g + 8 * (lane >> 5) + e;
      const float* const act = m.act + (size_t)(at < t1 ? (a.perm ? a.perm[at] : at) : 0) * a.rank;
#pragma unroll
      for (int j = 0; j < RB; ++j) {
        const int r = 32 * j + (lane & 31);
        _Float16 h, l;
        split2(at < t1 && r < a.rank ? act[r] * up : 0.0f, h, l);
        hi[j][e] = h;
        lo[j][e] = l;
      }
    }
    wave_fence();
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      const half8 v = read_transposed(mine, kFactorRow, 0, 32 * i);
#pragma unroll
      for (int j = 0; j < RB; ++j) {
        acc[j][i] = __builtin_amdgcn_mfma_f32_32x32x16_f16(hi[j], v, acc[j][i], 0, 0, 0);
        acc[j][i] = __builtin_amdgcn_mfma_f32_32x32x16_f16(lo[j], v, acc[j][i], 0, 0, 0);
      }
    }
    wave_fence();
  }

  const float by = down * a.scale[adapter];
  float* const red = reinterpret_cast<float*>(lds);  // [wave][column block][register][lane]
  float* const out = m.out + ((size_t)blockIdx.y * a.count + adapter) * a.rank * m.width;
#pragma unroll
  for (int j = 0; j < RB; ++j) {
    __syncthreads();
#pragma unroll
    for (int i = 0; i < 2; ++i)
#pragma unroll
      for (int e = 0; e < 16; ++e) red[((wave * 2 + i) * 16 + e) * 64 + lane] = acc[j][i][e];
    __syncthreads();
    // a wave adds eight of the 32 (block, register) pairs
#pragma unroll
    for (int q = 0; q < 8; ++q) {
      const int i = q & 1, e = 4 * wave + (q >> 1);
      float sum = red[(i * 16 + e) * 64 + lane];
#pragma unroll
      for (int w = 1; w < kWaves; ++w) sum += red[((w * 2 + i) * 16 + e) * 64 + lane];
      const int r = 32 * j + 8 * (e >> 2) + 4 * (lane >> 5) + (e & 3);
      const int f = f0 + 32 * i + (lane & 31);
      if (r < a.rank && f < m.width) out[(size_t)r * m.width + f] = by * sum;
    }
  }
}

struct ReduceArgs {
  const float* part[2];
  float* out[2];
  long long n[2];
  int splits;
};

__global__ __launch_bounds__(kThreads) void outer_reduce_kernel(ReduceArgs a) {
  const int y = blockIdx.y;
  const long long n = a.n[y];
  const long long stride = (long long)gridDim.x * kThreads;
  for (long long i = (long long)blockIdx.x * kThreads + threadIdx.x; i < n; i += stride) {
    float sum = a.part[y][i];
    for (int s = 1; s < a.splits; ++s) sum += a.part[y][(size_t)s * n + i];
    a.out[y][i] = sum;
  }
}

// ---------------------------------------------------------------------------
// Sort: one workgroup, stable, so that sums over an adapter's tokens have one
// order. Each of the 16 waves counts its part of the tokens; the counts'
// prefix sums over adapters, and over the waves of one adapter, give each
// wave's places; then the wave places its tokens 64 at a time, lanes of one
// adapter by their number. Bucket `count`: tokens without an adapter.

constexpr int kSortThreads = 1024;
constexpr int kSortWaves = kSortThreads / 64;

__global__ __launch_bounds__(kSortThreads) void sort_kernel(const int* ids, int n, int count, int* perm, int* first,
                                                            Tile* tiles, int max_tiles) {
  extern __shared__ int cnt[];  // [wave][bucket], then [bucket] first token and [bucket] first tile
  __shared__ int sums[2][kSortWaves];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int buckets = count + 1;
  int* const base = cnt + kSortWaves * buckets;
  int* const tile0 = base + buckets;
  const int per = (n + kSortThreads - 1) / kSortThreads * 64;
  const int i0 = min(n, wave * per), i1 = min(n, i0 + per);
  auto bucket = [&](int i) {
    const int id = ids[i];
    return (unsigned)id < (unsigned)count ? id : count;
  };
  for (int q = threadIdx.x; q < kSortWaves * buckets; q += kSortThreads) cnt[q] = 0;
  __syncthreads();
  for (int i = i0 + lane; i < i1; i += 64) atomicAdd(&cnt[wave * buckets + bucket(i)], 1);
  __syncthreads();
  // every thread owns `own` buckets in sequence
  const int own = (buckets + kSortThreads - 1) / kSortThreads;
  const int b0 = min(buckets, (int)threadIdx.x * own), b1 = min(buckets, b0 + own);
  int tokens = 0, n_tiles = 0;
  for (int b = b0; b < b1; ++b) {
    int sum = 0;
    for (int w = 0; w < kSortWaves; ++w) {
      const int c = cnt[w * buckets + b];
      cnt[w * buckets + b] = sum;
      sum += c;
    }
    base[b] = tokens;
    tile0[b] = n_tiles;
    tokens += sum;
    n_tiles += (sum + kTile - 1) / kTile;
  }
  int st = tokens, sl = n_tiles;
#pragma unroll
  for (int d = 1; d < 64; d <<= 1) {
    const int x = __shfl_up(st, d), y = __shfl_up(sl, d);
    if (lane >= d) {
      st += x;
      sl += y;
    }
  }
  if (lane == 63) {
    sums[0][wave] = st;
    sums[1][wave] = sl;
  }
  __syncthreads();
  int before_t = st - tokens, before_l = sl - n_tiles, all_tiles = 0;
  for (int w = 0; w < kSortWaves; ++w) {
    if (w < wave) {
      before_t += sums[0][w];
      before_l += sums[1][w];
    }
    all_tiles += sums[1][w];
  }
  for (int b = b0; b < b1; ++b) {
    base[b] += before_t;
    tile0[b] += before_l;
    first[b] = base[b];
  }
  if (threadIdx.x == 0) first[buckets] = n;
  __syncthreads();
  for (int b = wave; b < buckets; b += kSortWaves) {
    const int end = b + 1 < buckets ? base[b + 1] : n;
    const int of = (end - base[b] + kTile - 1) / kTile;
    for (int q = lane; q < of; q += 64)
      tiles[tile0[b] + q] = Tile{b < count ? b : -1, base[b] + q * kTile, min(kTile, end - base[b] - q * kTile), 0};
  }
  for (int q = all_tiles + threadIdx.x; q < max_tiles; q += kSortThreads) tiles[q] = Tile{-1, 0, 0, 0};
  int bits = 0;
  while ((1 << bits) < buckets) ++bits;
  for (int c = i0; c < i1; c += 64) {
    const bool in = c + lane < i1;
    const int b = in ? bucket(c + lane) : 0;
    uint64_t same = __ballot(in);
    for (int k = 0; k < bits; ++k) {
      const uint64_t set = __ballot(b >> k & 1);
      same &= (b >> k & 1) ? set : ~set;
    }
    if (in) {
      int* const mine = &cnt[wave * buckets + b];
      const int at = base[b] + *mine;
      const int rank = __popcll(same & ((1ull << lane) - 1));
      perm[at + rank] = c + lane;
      wave_fence();
      if (rank == 0) *mine += (int)__popcll(same);
    }
    wave_fence();
  }
}

// ---------------------------------------------------------------------------
// Host side.

using spdp::fail;

int hip_fail(hipError_t e, const char* what) {
  return fail(SPDP_ERR_HIP, std::string(what) + ": " + hipGetErrorString(e));
}

size_t aligned(size_t bytes) { return (bytes + 255) / 256 * 256; }

int compute_units(int* cus) {
  int dev = -1;
  hipError_t e = hipGetDevice(&dev);
  if (e != hipSuccess) return hip_fail(e, "hipGetDevice");
  e = hipDeviceGetAttribute(cus, hipDeviceAttributeMultiprocessorCount, dev);
  if (e != hipSuccess) return hip_fail(e, "hipDeviceGetAttribute");
  *cus = std::max(1, *cus);
  return SPDP_OK;
}

// The ranges of the width that shrink_kernel's workgroups take: about two
// workgroups per CU, at least 16 steps each (four per wave).
struct Ranges {
  int per, splits;
};
Ranges shrink_ranges(int64_t width, long long tiles, int banks, int cus) {
  const int steps = (int)((width + kStep - 1) / kStep);
  const int most = std::max(1, std::min(16, steps / 16));
  const int want = (int)std::min<long long>(most, std::max<long long>(1, 2 * cus / (tiles * banks)));
  const int per = (steps + want - 1) / want;
  return {per, (steps + per - 1) / per};
}

// The token pieces of outer_kernel, about two workgroups per CU, at least 64
// tokens each.
int outer_splits(const spdp_adapters_t* m, long long n_tokens, int cus) {
  const long long wgs = ((m->rows + kCols - 1) / kCols + (m->cols + kCols - 1) / kCols) * m->count;
  const long long want = std::max<long long>(1, 2 * cus / wgs);
  return (int)std::min<long long>({want, 16, std::max<long long>(1, n_tokens / m->count / 64)});
}

// What the sort writes, and where, and the launch's tiles.
struct SortPlan {
  bool sorted;
  long long tiles;  // of the grid
  size_t bytes;     // perm, first, tiles
};
SortPlan plan_sort(long long n_tokens, int count, bool ids, bool always) {
  SortPlan p;
  p.sorted = ids && (always || n_tokens > kSmall);
  p.tiles = !ids ? (n_tokens + kTile - 1) / kTile
            : p.sorted ? n_tokens / kTile + std::min<long long>(count + 1, n_tokens) + 1
                       : n_tokens;
  p.bytes = p.sorted ? aligned((size_t)n_tokens * 4) + aligned((size_t)(count + 2) * 4) + aligned((size_t)p.tiles * sizeof(Tile)) : 0;
  return p;
}

int check_bank(const spdp_adapters_t* m, const char* who) {
  const std::string s(who);
  if (!m->a || !m->b || !m->scale) return fail(SPDP_ERR_INVALID_ARG, s + ": a, b or scale is NULL");
  if (m->rows < 1 || m->cols < 1 || m->count < 1 || m->rank < 1)
    return fail(SPDP_ERR_INVALID_ARG, s + ": rows, cols, count and rank must be >= 1");
  if (m->rank > kMaxRank) return fail(SPDP_ERR_UNSUPPORTED, s + ": rank above 128");
  if (m->count > kMaxAdapters) return fail(SPDP_ERR_UNSUPPORTED, s + ": more than 2048 adapters");
  if (m->rows > 1 << 24 || m->cols > 1 << 24) return fail(SPDP_ERR_UNSUPPORTED, s + ": more than 2^24 rows or columns");
  return SPDP_OK;
}

int check_tokens(int64_t n_tokens) {
  if (n_tokens < 1) return fail(SPDP_ERR_INVALID_ARG, "n_tokens must be at least 1");
  if (n_tokens > 1 << 20) return fail(SPDP_ERR_UNSUPPORTED, "more than 2^20 tokens");
  return SPDP_OK;
}

bool overlap(const void* p, size_t np, const void* q, size_t nq) {
  const uintptr_t a = reinterpret_cast<uintptr_t>(p), b = reinterpret_cast<uintptr_t>(q);
  return a < b + nq && b < a + np;
}

// fp32 of the rank activations' partial sums
size_t part_bytes(long long n_tokens, int rank, int splits) { return aligned((size_t)splits * n_tokens * rank * 4); }

int sort_tokens(const int32_t* ids, long long n, int count, const SortPlan& p, unsigned char* ws, Tokens* t, int** first,
                hipStream_t st) {
  int* const perm = reinterpret_cast<int*>(ws);
  *first = reinterpret_cast<int*>(ws + aligned((size_t)n * 4));
  Tile* const tiles = reinterpret_cast<Tile*>(ws + aligned((size_t)n * 4) + aligned((size_t)(count + 2) * 4));
  const int lds = (kSortWaves + 2) * (count + 1) * 4;
  if (lds > 64 * 1024) {
    const hipError_t e =
        hipFuncSetAttribute(reinterpret_cast<const void*>(sort_kernel), hipFuncAttributeMaxDynamicSharedMemorySize, lds);
    if (e != hipSuccess) return hip_fail(e, "hipFuncSetAttribute");
  }
  hipLaunchKernelGGL(sort_kernel, dim3(1), dim3(kSortThreads), lds, st, ids, (int)n, count, perm, *first, tiles, (int)p.tiles);
  const hipError_t e = hipGetLastError();
  if (e != hipSuccess) return hip_fail(e, "kernel launch");
  t->perm = perm;
  t->tiles = tiles;
  return SPDP_OK;
}

template <int RB>
hipError_t launch_shrink_rb(const ShrinkArgs& a, dim3 grid, hipStream_t st) {
  hipLaunchKernelGGL(shrink_kernel<RB>, grid, dim3(kThreads), kWaves * kTile * 16 * RB * 4, st, a);
  return hipGetLastError();
}
hipError_t launch_shrink(const ShrinkArgs& a, dim3 grid, hipStream_t st) {
  if (a.rank <= 16) return launch_shrink_rb<1>(a, grid, st);
  if (a.rank <= 32) return launch_shrink_rb<2>(a, grid, st);
  if (a.rank <= 64) return launch_shrink_rb<4>(a, grid, st);
  return launch_shrink_rb<8>(a, grid, st);
}

template <int RB>
hipError_t launch_expand_rb(const ExpandArgs& a, dim3 grid, hipStream_t st) {
  const int lds = ExpandCfg<RB>::kLds;
  if (lds > 64 * 1024) {
    const hipError_t e = hipFuncSetAttribute(reinterpret_cast<const void*>(expand_kernel<RB>),
                                             hipFuncAttributeMaxDynamicSharedMemorySize, lds);
    if (e != hipSuccess) return e;
  }
  hipLaunchKernelGGL(expand_kernel<RB>, grid, dim3(kThreads), lds, st, a);
  return hipGetLastError();
}
hipError_t launch_expand(ExpandArgs& a, int banks, long long tiles, int cus, hipStream_t st) {
  int widest = 0;
  for (int i = 0; i < banks; ++i) widest = std::max(widest, a.m[i].width);
  const int blocks = (widest + kBlock - 1) / kBlock;
  // a workgroup keeps its tokens' activations for several blocks where that
  // leaves eight workgroups per CU
  a.blocks = (int)std::max<long long>(1, std::min<long long>(8, blocks * tiles * banks / (8ll * cus)));
  const dim3 grid((unsigned)((blocks + a.blocks - 1) / a.blocks), (unsigned)tiles, (unsigned)banks);
  if (a.rank <= 16) return launch_expand_rb<1>(a, grid, st);
  if (a.rank <= 32) return launch_expand_rb<2>(a, grid, st);
  if (a.rank <= 64) return launch_expand_rb<4>(a, grid, st);
  return launch_expand_rb<8>(a, grid, st);
}

hipError_t launch_outer(const OuterArgs& a, int widest, hipStream_t st) {
  const dim3 grid((unsigned)((widest + kCols - 1) / kCols), (unsigned)a.splits, (unsigned)(2 * a.count));
  if (a.rank <= 32)
    hipLaunchKernelGGL(outer_kernel<1>, grid, dim3(kThreads), 0, st, a);
  else if (a.rank <= 64)
    hipLaunchKernelGGL(outer_kernel<2>, grid, dim3(kThreads), 0, st, a);
  else
    hipLaunchKernelGGL(outer_kernel<4>, grid, dim3(kThreads), 0, st, a);
  return hipGetLastError();
}

int check_banks(const spdp_adapters_t* banks, int32_t n_banks, int64_t n_tokens) {
  if (!banks) return fail(SPDP_ERR_INVALID_ARG, "banks is NULL");
  if (n_banks < 1 || n_banks > kMaxBanks) return fail(SPDP_ERR_INVALID_ARG, "the number of banks must lie in [1, 8]");
  int st = check_tokens(n_tokens);
  if (st != SPDP_OK) return st;
  for (int i = 0; i < n_banks; ++i) {
    st = check_bank(&banks[i], "bank");
    if (st != SPDP_OK) return st;
    if (banks[i].rank != banks[0].rank || banks[i].count != banks[0].count)
      return fail(SPDP_ERR_INVALID_ARG, "the banks of one call must have one rank and one count");
  }
  return SPDP_OK;
}

struct AdaptPlan {
  SortPlan sort;
  Ranges r[kMaxBanks];
  int splits;  // the most of them
  size_t bytes;
};
void plan_adapt(const spdp_adapters_t* banks, int n_banks, long long n_tokens, bool ids, int cus, AdaptPlan* p) {
  p->sort = plan_sort(n_tokens, banks[0].count, ids, false);
  p->bytes = p->sort.bytes;
  p->splits = 1;
  for (int i = 0; i < n_banks; ++i) {
    p->r[i] = shrink_ranges(banks[i].cols, p->sort.tiles, n_banks, cus);
    p->splits = std::max(p->splits, p->r[i].splits);
    p->bytes += part_bytes(n_tokens, banks[i].rank, p->r[i].splits);
  }
}

struct GradPlan {
  SortPlan sort;
  Ranges r;
  int splits;
  size_t part, u, outer[2], bytes;
};
void plan_grad(const spdp_adapters_t* m, long long n_tokens, bool ids, int cus, GradPlan* p) {
  p->sort = plan_sort(n_tokens, m->count, ids, true);
  p->r = shrink_ranges(m->rows, p->sort.tiles, 1, cus);
  p->splits = outer_splits(m, n_tokens, cus);
  p->part = part_bytes(n_tokens, m->rank, p->r.splits);
  p->u = part_bytes(n_tokens, m->rank, 1);
  const size_t each = (size_t)p->splits * m->count * m->rank * 4;
  p->outer[0] = p->splits > 1 ? aligned(each * m->cols) : 0;
  p->outer[1] = p->splits > 1 ? aligned(each * m->rows) : 0;
  p->bytes = p->sort.bytes + p->part + p->u + p->outer[0] + p->outer[1];
}

int check_workspace(const void* workspace, size_t have, size_t need) {
  if (!workspace) return fail(SPDP_ERR_INVALID_ARG, "workspace is NULL");
  if (reinterpret_cast<uintptr_t>(workspace) & 255) return fail(SPDP_ERR_INVALID_ARG, "workspace must be 256-byte aligned");
  if (have < need)
    return fail(SPDP_ERR_INVALID_ARG, "workspace of " + std::to_string(have) + " bytes, " + std::to_string(need) + " needed");
  return SPDP_OK;
}

int adapt_workspace(const spdp_adapters_t* banks, int32_t n_banks, int64_t n_tokens, int32_t with_ids, size_t* bytes) {
  int st = check_banks(banks, n_banks, n_tokens);
  int cus = 1;
  if (st == SPDP_OK) st = compute_units(&cus);
  if (st != SPDP_OK) return st;
  AdaptPlan p;
  plan_adapt(banks, n_banks, n_tokens, with_ids != 0, cus, &p);
  *bytes = p.bytes;
  return SPDP_OK;
}

int adapt(const spdp_adapters_t* banks, int32_t n_banks, const uint16_t* const* X, const int32_t* ids,
          const uint16_t* const* base, uint16_t* const* Y, float* const* H, int64_t n_tokens, void* workspace,
          size_t workspace_bytes, void* stream) {
  int st = check_banks(banks, n_banks, n_tokens);
  if (st != SPDP_OK) return st;
  if (!X || !base || !Y) return fail(SPDP_ERR_INVALID_ARG, "X, base or Y is NULL");
  const size_t n = (size_t)n_tokens;
  for (int i = 0; i < n_banks; ++i) {
    if (!X[i] || !base[i] || !Y[i] || (H && !H[i])) return fail(SPDP_ERR_INVALID_ARG, "X, base, Y or H of a bank is NULL");
    const size_t out = n * banks[i].rows * 2, kept = n * banks[i].rank * 4;
    for (int j = 0; j < n_banks; ++j) {
      const size_t in = n * banks[j].cols * 2, other = n * banks[j].rows * 2;
      if (overlap(Y[i], out, X[j], in)) return fail(SPDP_ERR_INVALID_ARG, "an output overlaps an input");
      if (overlap(Y[i], out, base[j], other) && !(i == j && Y[i] == base[j]))
        return fail(SPDP_ERR_INVALID_ARG, "an output overlaps a base other than its own as a whole");
      if (i != j && overlap(Y[i], out, Y[j], other)) return fail(SPDP_ERR_INVALID_ARG, "outputs overlap");
      if (H && (overlap(H[i], kept, X[j], in) || overlap(H[i], kept, base[j], other) || overlap(H[i], kept, Y[j], other) ||
                (i != j && overlap(H[i], kept, H[j], kept))))
        return fail(SPDP_ERR_INVALID_ARG, "H overlaps another array");
    }
  }
  int cus = 1;
  st = compute_units(&cus);
  if (st != SPDP_OK) return st;
  AdaptPlan p;
  plan_adapt(banks, n_banks, n_tokens, ids != nullptr, cus, &p);
  st = check_workspace(workspace, workspace_bytes, p.bytes);
  if (st != SPDP_OK) return st;

  auto s = static_cast<hipStream_t>(stream);
  Tokens t = {ids, nullptr, nullptr, (int)n_tokens, banks[0].count};
  unsigned char* ws = static_cast<unsigned char*>(workspace);
  if (p.sort.sorted) {
    int* first;
    st = sort_tokens(ids, n_tokens, banks[0].count, p.sort, ws, &t, &first, s);
    if (st != SPDP_OK) return st;
    ws += p.sort.bytes;
  }
  ShrinkArgs sa;
  ExpandArgs ea;
  std::memset(&sa, 0, sizeof(sa));
  std::memset(&ea, 0, sizeof(ea));
  sa.t = ea.t = t;
  sa.rank = ea.rank = banks[0].rank;
  for (int i = 0; i < n_banks; ++i) {
    const spdp_adapters_t& b = banks[i];
    float* const part = reinterpret_cast<float*>(ws);
    ws += part_bytes(n_tokens, b.rank, p.r[i].splits);
    sa.m[i] = Shrink{X[i], b.a, part, (int)b.cols, p.r[i].per};
    ea.m[i] = Expand{part, b.b, b.scale, base[i], Y[i], H ? H[i] : nullptr, (int)b.rows, p.r[i].splits};
  }
  hipError_t e = launch_shrink(sa, dim3((unsigned)p.sort.tiles, (unsigned)p.splits, (unsigned)n_banks), s);
  if (e == hipSuccess) e = launch_expand(ea, n_banks, p.sort.tiles, cus, s);
  return e == hipSuccess ? SPDP_OK : hip_fail(e, "kernel launch");
}

int adapt_grad_workspace(const spdp_adapters_t* bank, int64_t n_tokens, int32_t with_ids, size_t* bytes) {
  int st = check_banks(bank, 1, n_tokens);
  int cus = 1;
  if (st == SPDP_OK) st = compute_units(&cus);
  if (st != SPDP_OK) return st;
  GradPlan p;
  plan_grad(bank, n_tokens, with_ids != 0, cus, &p);
  *bytes = p.bytes;
  return SPDP_OK;
}

int adapt_grad(const spdp_adapters_t* bank, const uint16_t* X, const int32_t* ids, const float* H, const uint16_t* dY,
               const uint16_t* base, uint16_t* dX, float* dA, float* dB, int64_t n_tokens, void* workspace,
               size_t workspace_bytes, void* stream) {
  int st = check_banks(bank, 1, n_tokens);
  if (st != SPDP_OK) return st;
  if (!X || !H || !dY || !base || !dX || !dA || !dB) return fail(SPDP_ERR_INVALID_ARG, "an array is NULL");
  const size_t n = (size_t)n_tokens, fac = (size_t)bank->count * bank->rank;
  const struct {
    const void* p;
    size_t bytes;
  } in[] = {{X, n * bank->cols * 2}, {H, n * bank->rank * 4}, {dY, n * bank->rows * 2}, {base, n * bank->cols * 2},
            {bank->a, fac * bank->cols * 2}, {bank->b, fac * bank->rows * 2}},
    out[] = {{dX, n * bank->cols * 2}, {dA, fac * bank->cols * 4}, {dB, fac * bank->rows * 4}};
  for (const auto& o : out) {
    for (const auto& i : in)
      if (overlap(o.p, o.bytes, i.p, i.bytes) && !(&o == &out[0] && &i == &in[3] && i.p == o.p))
        return fail(SPDP_ERR_INVALID_ARG, "an output overlaps an input (dX may be its base as a whole)");
    for (const auto& q : out)
      if (&q != &o && overlap(o.p, o.bytes, q.p, q.bytes)) return fail(SPDP_ERR_INVALID_ARG, "outputs overlap");
  }
  int cus = 1;
  st = compute_units(&cus);
  if (st != SPDP_OK) return st;
  GradPlan p;
  plan_grad(bank, n_tokens, ids != nullptr, cus, &p);
  st = check_workspace(workspace, workspace_bytes, p.bytes);
  if (st != SPDP_OK) return st;

  auto s = static_cast<hipStream_t>(stream);
  unsigned char* ws = static_cast<unsigned char*>(workspace);
  Tokens t = {ids, nullptr, nullptr, (int)n_tokens, bank->count};
  int* first = nullptr;
  if (p.sort.sorted) {
    st = sort_tokens(ids, n_tokens, bank->count, p.sort, ws, &t, &first, s);
    if (st != SPDP_OK) return st;
    ws += p.sort.bytes;
  }
  float* const part = reinterpret_cast<float*>(ws);
  float* const u = reinterpret_cast<float*>(ws + p.part);
  float* const pa = reinterpret_cast<float*>(ws + p.part + p.u);
  float* const pb = reinterpret_cast<float*>(ws + p.part + p.u + p.outer[0]);
  ShrinkArgs sa;
  ExpandArgs ea;
  OuterArgs oa;
  std::memset(&sa, 0, sizeof(sa));
  std::memset(&ea, 0, sizeof(ea));
  std::memset(&oa, 0, sizeof(oa));
  sa.t = ea.t = t;
  sa.rank = ea.rank = oa.rank = bank->rank;
  sa.m[0] = Shrink{dY, bank->b, part, (int)bank->rows, p.r.per};
  ea.m[0] = Expand{part, bank->a, bank->scale, base, dX, u, (int)bank->cols, p.r.splits};
  hipError_t e = launch_shrink(sa, dim3((unsigned)p.sort.tiles, (unsigned)p.r.splits, 1), s);
  if (e == hipSuccess) e = launch_expand(ea, 1, p.sort.tiles, cus, s);
  if (e != hipSuccess) return hip_fail(e, "kernel launch");
  const bool split = p.splits > 1;
  oa.m[0] = Outer{u, X, split ? pa : dA, (int)bank->cols};
  oa.m[1] = Outer{H, dY, split ? pb : dB, (int)bank->rows};
  oa.scale = bank->scale;
  oa.perm = t.perm;
  oa.first = first;
  oa.n_tokens = (int)n_tokens;
  oa.count = bank->count;
  oa.splits = p.splits;
  e = launch_outer(oa, (int)std::max(bank->rows, bank->cols), s);
  if (e == hipSuccess && split) {
    ReduceArgs ra;
    std::memset(&ra, 0, sizeof(ra));
    ra.part[0] = pa;
    ra.part[1] = pb;
    ra.out[0] = dA;
    ra.out[1] = dB;
    ra.n[0] = (long long)fac * bank->cols;
    ra.n[1] = (long long)fac * bank->rows;
    ra.splits = p.splits;
    const unsigned blocks = (unsigned)std::min<long long>(2048, (std::max(ra.n[0], ra.n[1]) + kThreads - 1) / kThreads);
    hipLaunchKernelGGL(outer_reduce_kernel, dim3(blocks, 2), dim3(kThreads), 0, s, ra);
    e = hipGetLastError();
  }
  return e == hipSuccess ? SPDP_OK : hip_fail(e, "kernel launch");
}

// No C++ exception leaves the ABI: a message may find no memory.
template <class F>
int guarded(F f) {
  try {
    spdp::clear_error();
    return f();
  } catch (...) {
    return SPDP_ERR_OOM;
  }
}

}  // namespace

extern "C" {

int spdp_adapt_workspace(const spdp_adapters_t* banks, int32_t n_banks, int64_t n_tokens, int32_t with_ids, size_t* bytes) {
  return guarded([&] {
    if (!bytes) return fail(SPDP_ERR_INVALID_ARG, "bytes is NULL");
    return adapt_workspace(banks, n_banks, n_tokens, with_ids, bytes);
  });
}

int spdp_adapt(const spdp_adapters_t* banks, int32_t n_banks, const uint16_t* const* X, const int32_t* ids,
               const uint16_t* const* base, uint16_t* const* Y, float* const* H, int64_t n_tokens, void* workspace,
               size_t workspace_bytes, void* stream) {
  return guarded([&] { return adapt(banks, n_banks, X, ids, base, Y, H, n_tokens, workspace, workspace_bytes, stream); });
}

int spdp_adapt_grad_workspace(const spdp_adapters_t* bank, int64_t n_tokens, int32_t with_ids, size_t* bytes) {
  return guarded([&] {
    if (!bytes) return fail(SPDP_ERR_INVALID_ARG, "bytes is NULL");
    return adapt_grad_workspace(bank, n_tokens, with_ids, bytes);
  });
}

int spdp_adapt_grad(const spdp_adapters_t* bank, const uint16_t* X, const int32_t* ids, const float* H, const uint16_t* dY,
                    const uint16_t* base, uint16_t* dX, float* dA, float* dB, int64_t n_tokens, void* workspace,
                    size_t workspace_bytes, void* stream) {
  return guarded([&] {
    return adapt_grad(bank, X, ids, H, dY, base, dX, dA, dB, n_tokens, workspace, workspace_bytes, stream);
  });
}

}  // extern "C"
