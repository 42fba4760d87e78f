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
//   sort_kernel    tokens in the order of their adapters, and tiles of them, so
//                  that an MFMA's tokens share a factor.
//
// Both factors are kept rank by rank ([adapter][rank][width]): the backward
// pass is the forward one with the factors exchanged (u = B^T dY by
// shrink_kernel, s A^T u by expand_kernel).
//
// h and u are fp32. Where they are operands of fp16 MFMAs they are scaled by a
// power of two, so that the largest lies in [2^13, 2^14), and split into the
// nearest fp16 and the rest's nearest fp16: 22 bits or, for small ones, 2^-38
// of the largest. Two MFMAs instead of one; the launches are bound by memory.
// In the factors' gradients, which are fp32, the sums over up to kFew tokens take
// fp32 MFMAs instead.
//
// Measured, on a card that copies at 5.2 TB/s: shrink_kernel, 2048 tokens, 8192
// wide, rank 32, 11.2 us (34 MB of input, 3 TB/s, and the factor from L2);
// expand_kernel behind it, 28672 wide, 54 us (235 MB, 4.4 TB/s); outer_kernel, 4096
// tokens, 13824 + 5120 wide, rank 64, 41 us (155 MB, 3.8 TB/s); sort_kernel, 2048
// ids, 6 us, a chain of LDS round trips. Small calls are bound by the launches,
// 4 to 7 us each.

#include <hip/hip_fp16.h>
#include <hip/hip_runtime.h>

#include <algorithm>
#include <cstring>

#include "calls.h"
#include "lanes.h"
#include "lowrank.h"

namespace {

using namespace spdp_low;

using namespace spdp_dev;

typedef float float4v __attribute__((ext_vector_type(4)));

constexpr int kThreads = 256;
constexpr int kWaves = 4;

// The tokens of tile `block`, at most T, to tok[0 .. T - 1] (places past the
// count repeat one of them); false: no tile. Every wave does it alike.
// `subs`: T-token parts of the sort's tiles.
template <int T>
__device__ __forceinline__ bool take_tile(const Tokens& t, int block, int* tok, int& adapter, int& count, int subs = 1) {
  const int lane = threadIdx.x & 63;
  if (t.ids == nullptr) {
    adapter = 0;
    count = min(T, t.n_tokens - block * T);
    if (lane < T) tok[lane] = block * T + min(lane, count - 1);
  } else if (t.tiles == nullptr) {
    // the tile of token `block`, which has to be the first, (T + 1)st, ... of its adapter
    int id = lane < t.n_tokens ? t.ids[lane] : -2;
    if (id >= t.count || (lane < t.n_tokens && id < 0)) id = -1;
    adapter = __builtin_amdgcn_readlane(id, block);
    const uint64_t same = __ballot(lane < t.n_tokens && id == adapter);
    const int first = __popcll(same & ((1ull << block) - 1));
    if (first % T != 0) return false;
    count = min(T, (int)__popcll(same) - first);
    const int rank = (int)__popcll(same & ((1ull << lane) - 1)) - first;
    if ((same >> lane & 1) && rank >= 0 && rank < T) tok[rank] = lane;
    if (lane >= count && lane < T) tok[lane] = block;
  } else {
    const Tile d = t.tiles[block / subs];
    const int skip = block % subs * T;
    adapter = d.adapter;
    count = min(T, d.count - skip);
    if (count <= 0) return false;
    if (lane < T) tok[lane] = t.perm[d.start + skip + min(lane, count - 1)];
  }
  wave_fence();
  return true;
}

// ---------------------------------------------------------------------------
// Shrink. A workgroup owns a tile of tokens and a range of the width, its four (or
// eight) waves every fourth (eighth) step of 64 columns; 16x16x32 MFMAs with the tokens as
// rows. The waves' sums are added in LDS.

constexpr int kStep = 64;

// The sums over the steps [s0, s1) of in's rows tok[0 .. T - 1] times the
// adapter's factor, each of W waves' share to red [wave][token][16 RB].
template <int RB, int T, int W>
__device__ __forceinline__ void shrink_steps(const uint16_t* in, const uint16_t* factor, int width, int rank, const int* tok,
                                             int s0, int s1, float* red) {
  constexpr int TB = T / 16;
  // halves of a step that are loaded at once, the next ones during their MFMAs
  constexpr int D = RB + TB <= 5 ? 4 : RB + TB <= 10 ? 2 : 1;
  const int lane = threadIdx.x & 63;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  // four lanes have a row's 64 columns, 16 of them each: 128 bytes of a row at
  // a time (in an order of the sum that both operands share)
  const int k0 = 16 * (lane >> 4);
  const uint16_t *px[TB], *pf[RB];
#pragma unroll
  for (int i = 0; i < TB; ++i) px[i] = in + (size_t)tok[16 * i + (lane & 15)] * width + k0;
#pragma unroll
  for (int j = 0; j < RB; ++j) pf[j] = factor + (size_t)min(16 * j + (lane & 15), rank - 1) * width + k0;

  float4v acc[TB][RB];
#pragma unroll
  for (int i = 0; i < TB; ++i)
#pragma unroll
    for (int j = 0; j < RB; ++j) acc[i][j] = float4v{0, 0, 0, 0};
  struct Halves {
    half8 x[D][TB], f[D][RB];
  };
  // from half h of the wave on; `whole`: all columns lie inside the width
  auto load = [&](int h, bool whole, Halves& b) __attribute__((always_inline)) {
#pragma unroll
    for (int d = 0; d < D; ++d) {
      const int at = (s0 + wave + ((h + d) >> 1) * W) * kStep + 8 * ((h + d) & 1);
      const int left = whole ? 8 : max(width - at - k0, 0);
#pragma unroll
      for (int i = 0; i < TB; ++i) b.x[d][i] = whole ? load8(px[i] + at) : load8_inside(px[i] + at, left);
#pragma unroll
      for (int j = 0; j < RB; ++j) b.f[d][j] = whole ? load8(pf[j] + at) : load8_inside(pf[j] + at, left);
    }
  };
  auto multiply = [&](const Halves& b) __attribute__((always_inline)) {
#pragma unroll
    for (int d = 0; d < D; ++d)
#pragma unroll
      for (int i = 0; i < TB; ++i)
#pragma unroll
        for (int j = 0; j < RB; ++j)
          acc[i][j] = __builtin_amdgcn_mfma_f32_16x16x32_f16(b.x[d][i], b.f[d][j], acc[i][j], 0, 0, 0);
  };
  // the wave's halves that lie inside the width, by batches of D, then the rest
  const int mine = max(0, (min(s1, width / kStep) - s0 - wave + W - 1) / W);
  const int inside = 2 * mine / D;
  Halves even, odd;
  int b = 0;
  if (b < inside) load(0, true, even);
  while (b < inside) {
    if (b + 1 < inside) load((b + 1) * D, true, odd);
    multiply(even);
    if (++b >= inside) break;
    if (b + 1 < inside) load((b + 1) * D, true, even);
    multiply(odd);
    ++b;
  }
  // (a step past the range, or columns past the width, load zeros)
  const int all = 2 * max(0, (s1 - s0 - wave + W - 1) / W);
  for (int h = inside * D; h < all; h += D) {
    if constexpr (D <= 2) {
      load(h, false, even);
    } else {
#pragma unroll
      for (int d = 0; d < D; ++d) {
        const int at = (s0 + wave + ((h + d) >> 1) * W) * kStep + 8 * ((h + d) & 1);
        const int left = h + d < all ? max(width - at - k0, 0) : 0;
#pragma unroll
        for (int i = 0; i < TB; ++i) even.x[d][i] = load8_inside(px[i] + at, left);
#pragma unroll
        for (int j = 0; j < RB; ++j) even.f[d][j] = load8_inside(pf[j] + at, left);
      }
    }
    multiply(even);
  }

  // register e of block (i, j): token 16 i + 4 (lane / 16) + e, rank 16 j + lane mod 16
#pragma unroll
  for (int i = 0; i < TB; ++i)
#pragma unroll
    for (int j = 0; j < RB; ++j)
#pragma unroll
      for (int e = 0; e < 4; ++e)
        red[((wave * T + 16 * i + 4 * (lane >> 4) + e) * RB + j) * 16 + (lane & 15)] = acc[i][j][e];
}

template <int RB, int T, int W>  // 16 RB ranks, tiles of T tokens, W waves
__global__ __launch_bounds__(64 * W) void shrink_kernel(ShrinkArgs a) {
  __shared__ int tok[T];
  extern __shared__ __attribute__((aligned(16))) float red[];  // [wave][token][16 RB]
  const Shrink& m = a.m[blockIdx.z];
  int adapter, count;
  if (!take_tile<T>(a.t, blockIdx.x, tok, adapter, count) || adapter < 0) return;
  const int steps = (m.width + kStep - 1) / kStep;
  const int s0 = (int)blockIdx.y * m.per;
  if (s0 >= steps) return;  // the grid has the most ranges of the launch's products
  shrink_steps<RB, T, W>(m.in, m.factor + (size_t)adapter * a.rank * m.width, m.width, a.rank, tok, s0,
                              min(steps, s0 + m.per), red);
  __syncthreads();
  float* const part = m.part + (size_t)blockIdx.y * a.t.n_tokens * a.rank;
  for (int q = threadIdx.x; q < count * 16 * RB; q += 64 * W) {
    const int t = q / (16 * RB), j = q % (16 * RB);
    if (j >= a.rank) continue;
    float sum = red[q];
#pragma unroll
    for (int w = 1; w < W; ++w) sum += red[w * T * 16 * RB + q];
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
constexpr int kFactorRow = 144;  // bytes of a factor row in LDS: 64 fp16 + 16, which spreads the rows over the banks
constexpr int kOutRow = 72;      // floats of a row of sums

// Few tokens and a small first factor: the fused form of eight waves computes h
// as well, every workgroup for itself, while its base and factor are on their
// way; one launch instead of two.

constexpr int kFusedWaves = 8;

template <int RB, int T, int W>
struct ExpandCfg {
  static constexpr int kRank = 16 * RB;
  static constexpr int kActRow = 2 * kRank + 16;  // bytes
  static constexpr int kPart = RB < 4 ? RB : 4;   // blocks of 16 ranks of the factor that are in LDS at a time
  static constexpr int kFactor = 16 * kPart * kFactorRow;
  static constexpr int kWave = kFactor > 4 * T * kOutRow ? kFactor : 4 * T * kOutRow;
  static constexpr int kActs = 32 * kActRow;  // (an MFMA reads 32 rows)
  static constexpr int kLds = 2 * kActs + W * kWave;
  static_assert(W != kFusedWaves || T * kRank * 4 <= kWave, "the waves' shares of h fit");
};

template <int RB, int T, bool FUSED, bool ONCE>  // 16 RB ranks, tiles of T <= 32 tokens; ONCE: past the caches
__global__ __launch_bounds__(64 * (FUSED ? kFusedWaves : kWaves)) void expand_kernel(ExpandArgs a) {
  constexpr int W = FUSED ? kFusedWaves : kWaves;
  constexpr int kBlock = kCols * W;
  using C = ExpandCfg<RB, T, W>;
  constexpr int kPasses = T / 8;  // of 8 tokens x 64 columns
  __shared__ int tok[T];
  __shared__ float mult[T];
  extern __shared__ __attribute__((aligned(16))) unsigned char lds[];
  const Expand& m = a.m[blockIdx.z];
  const int lane = threadIdx.x & 63;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  if ((int)blockIdx.x * kBlock >= m.width) return;
  int adapter, count;
  if (!take_tile<T>(a.t, blockIdx.y, tok, adapter, count, a.subs)) return;
  unsigned char* const act_hi = lds;
  unsigned char* const act_lo = lds + C::kActs;
  unsigned char* const mine = lds + 2 * C::kActs + wave * C::kWave;
  // neighbouring workgroups have neighbouring blocks at a time
  const int first = (int)blockIdx.x * kBlock + wave * kCols + 8 * (lane & 7);
  const int stride = (int)gridDim.x * kBlock;
  const uint16_t* const factor = m.factor + (size_t)max(adapter, 0) * a.rank * m.width;
  const float scale = m.scale[max(adapter, 0)];
  size_t row[kPasses];  // of the lane's tokens
#pragma unroll
  for (int p = 0; p < kPasses; ++p) row[p] = (size_t)tok[8 * p + (lane >> 3)] * m.width;

  const half8 none = half8{0, 0, 0, 0, 0, 0, 0, 0};
  // a block's base and factor, the latter by parts, requested a part ahead
  constexpr int kParts = RB / C::kPart;
  half8 base[kPasses], fac[2 * C::kPart];
  auto request = [&](int col, int part) __attribute__((always_inline)) {
    const int left = m.width - col;  // columns of the lane's eight that there are; may be negative
    if (left <= 0) return;
#pragma unroll
    for (int p = 0; p < kPasses; ++p)
      if (part == 0 && 8 * p + (lane >> 3) < count)
        base[p] = ONCE ? load8_once(m.base + row[p] + col, left) : load8_inside(m.base + row[p] + col, left);
    if (adapter < 0) return;
#pragma unroll
    for (int p = 0; p < 2 * C::kPart; ++p) {
      const int j = 16 * C::kPart * part + 8 * p + (lane >> 3);
      fac[p] = j < a.rank ? load8_inside(factor + (size_t)j * m.width + col, left) : none;
    }
  };
#pragma unroll
  for (int p = 0; p < kPasses; ++p) base[p] = none;
#pragma unroll
  for (int p = 0; p < 2 * C::kPart; ++p) fac[p] = none;
  request(first, 0);

  float* const red = reinterpret_cast<float*>(lds + 2 * C::kActs);
  if constexpr (FUSED) {
    if (adapter >= 0)
      shrink_steps<RB, T, W>(m.in, m.first_factor + (size_t)adapter * a.rank * m.in_width, m.in_width, a.rank, tok, 0,
                             (m.in_width + kStep - 1) / kStep, red);
    __syncthreads();
  }
  const int part8 = threadIdx.x & 7;  // eight threads a token
  const bool lead = blockIdx.x == 0;
  const int t = threadIdx.x >> 3;
  if (t < T) {
    const uint32_t at0 = (uint32_t)tok[t] * (uint32_t)a.rank;  // (2^20 tokens, 128 ranks at most)
    if (adapter >= 0) {
      const size_t plane = (size_t)a.t.n_tokens * a.rank;
      float v[2 * RB];
      float largest = 0.0f;
#pragma unroll
      for (int i = 0; i < 2 * RB; ++i) v[i] = 0.0f;
      if constexpr (FUSED) {
#pragma unroll
        for (int w = 0; w < W; ++w)
#pragma unroll
          for (int i = 0; i < 2 * RB; ++i) v[i] += red[(w * T + t) * C::kRank + 8 * i + part8];
#pragma unroll
        for (int i = 0; i < 2 * RB; ++i)  // (ranks that are none repeat the last)
          if (8 * i + part8 >= a.rank) v[i] = 0.0f;
      } else {
        // all ranks of some ranges in flight, added in order
        constexpr int S = RB >= 4 ? 2 : 8 / RB;
        for (int s0 = 0; s0 < m.splits; s0 += S) {
          float x[S][2 * RB];
#pragma unroll
          for (int s = 0; s < S; ++s)
#pragma unroll
            for (int i = 0; i < 2 * RB; ++i)
              x[s][i] = (m.part + min(s0 + s, m.splits - 1) * plane)[at0 + (uint32_t)min(8 * i + part8, a.rank - 1)];
#pragma unroll
          for (int s = 0; s < S; ++s)
#pragma unroll
            for (int i = 0; i < 2 * RB; ++i) v[i] += s0 + s < m.splits && 8 * i + part8 < a.rank ? x[s][i] : 0.0f;
        }
      }
#pragma unroll
      for (int i = 0; i < 2 * RB; ++i) {
        const int j = 8 * i + part8;
        if (m.keep != nullptr && lead && t < count && j < a.rank) m.keep[at0 + j] = v[i];
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
        const int at = t * C::kActRow + 2 * (8 * i + part8);
        *reinterpret_cast<_Float16*>(act_hi + at) = hi;
        *reinterpret_cast<_Float16*>(act_lo + at) = lo;
      }
      if (part8 == 0) {
        mult[t] = down * scale;
        if (m.most != nullptr && lead && t < count) m.most[tok[t]] = largest;
      }
      if (m.most != nullptr && lead && t < count) {
        float other = 0.0f;
#pragma unroll
        for (int i = 0; i < 2 * RB; ++i) other = fmaxf(other, finite_abs(m.other[at0 + (uint32_t)min(8 * i + part8, a.rank - 1)]));
#pragma unroll
        for (int d = 1; d < 8; d <<= 1) other = fmaxf(other, __shfl_xor(other, d));
        if (part8 == 0) m.most[a.t.n_tokens + tok[t]] = other;
      }
    } else if (m.keep != nullptr && lead && t < count) {
      for (int j = part8; j < a.rank; j += 8) m.keep[at0 + j] = 0.0f;
    }
  }
  __syncthreads();

  for (int b = 0; b < a.blocks; ++b) {
    const int col = first + b * stride;
    if (col - 8 * (lane & 7) >= m.width) return;
    const int left = m.width - col;
    half8 mybase[kPasses];
#pragma unroll
    for (int p = 0; p < kPasses; ++p) mybase[p] = base[p];
    float* const sums = reinterpret_cast<float*>(mine);
    if (adapter < 0 && b + 1 < a.blocks) request(col + stride, 0);
    if (adapter >= 0) {
      float16v acc[2] = {float16v{}, float16v{}};
#pragma unroll
      for (int part = 0; part < kParts; ++part) {
#pragma unroll
        for (int p = 0; p < 2 * C::kPart; ++p)
          *reinterpret_cast<half8*>(mine + (8 * p + (lane >> 3)) * kFactorRow + 16 * (lane & 7)) = left > 0 ? fac[p] : none;
        if (part + 1 < kParts)
          request(col, part + 1);
        else if (b + 1 < a.blocks)
          request(col + stride, 0);
        wave_fence();
#pragma unroll
        for (int k = 0; k < C::kPart; ++k) {
          const int at = (lane & 31) * C::kActRow + 2 * (16 * (C::kPart * part + k) + 8 * (lane >> 5));
          const half8 hi = *reinterpret_cast<const half8*>(act_hi + at), lo = *reinterpret_cast<const half8*>(act_lo + at);
#pragma unroll
          for (int i = 0; i < 2; ++i) {
            const half8 v = read_transposed(mine, kFactorRow, 16 * k, 32 * i);
            acc[i] = __builtin_amdgcn_mfma_f32_32x32x16_f16(hi, v, acc[i], 0, 0, 0);
            acc[i] = __builtin_amdgcn_mfma_f32_32x32x16_f16(lo, v, acc[i], 0, 0, 0);
          }
        }
        wave_fence();
      }
      // register e: token 8 (e / 4) + 4 (lane / 32) + e mod 4, column lane mod 32
#pragma unroll
      for (int i = 0; i < 2; ++i)
#pragma unroll
        for (int e = 0; e < T / 2; ++e)
          sums[(8 * (e >> 2) + 4 * (lane >> 5) + (e & 3)) * kOutRow + 32 * i + (lane & 31)] = acc[i][e];
      wave_fence();
    }
#pragma unroll
    for (int p = 0; p < kPasses; ++p) {
      const int q = 8 * p + (lane >> 3);
      if (q >= count || left <= 0) continue;
      half8 y = mybase[p];
      if (adapter >= 0) {
        const float* const sum = sums + q * kOutRow + 8 * (lane & 7);
        const float by = mult[q];
#pragma unroll
        for (int e = 0; e < 8; ++e) y[e] = (_Float16)__fmaf_rn(by, sum[e], (float)mybase[p][e]);
      }
      // (an output that the L2 caches cannot hold does not go through them, nor does
      // its base: whole passes, through them / the output past them / both, 2048 tokens,
      // 28672 wide, 80.4 / 77.8 / 75.5 us, 4000 tokens of 8 adapters, 8192 wide, the
      // latter two 66.7 / 60.8)
      if (ONCE && left >= 8) {
        typedef half8 half8_any __attribute__((aligned(2)));
        __builtin_nontemporal_store(y, reinterpret_cast<half8_any*>(m.out + row[p] + col));
      } else {
        store8_inside(m.out + row[p] + col, y, left);
      }
    }
    wave_fence();
  }
}

// ---------------------------------------------------------------------------
// Outer: for an adapter, out[j][f] = scale * sum over its tokens of act[t][j]
// in[t][f]. A piece is an adapter's tokens or, split, a part of them.
//
// An adapter of up to kFew tokens: fp32 MFMAs on the activations as they are (lane l
// has rank l mod 32 and the tokens 8 (l / 32) .. + 7, and of the input column l mod
// 32 and the same tokens, so step e of eight multiplies tokens e and 8 + e). In sums
// of so few products the 22 bits of two fp16 would show, and in ranks far below the
// others fewer; in sums of more the additions' own error is as large. A product takes
// the matrix cores eight times as long as those of the two fp16 (backward passes,
// 4096 x 4096, two fp16 / fp32: 32 tokens of rank 16 18.2 / 18.8 us, 64 of four
// adapters of rank 64 25.2 / 25.2, 2000 of 64 of rank 16 63.5 / 70).
//
// With few tokens in all outer_kernel makes the operands itself (DIRECT), a launch less.
// Else pack_kernel lays a piece's activations out as the MFMA's operands, scaled by
// one power of two (by each token's largest, which expand_kernel has left) and
// split into two fp16: [group of 16 tokens][block of 32
// ranks][high, low][lane][8]. outer_kernel's workgroup owns 64 columns, all
// ranks and a piece, each wave every fourth group (an MFMA's k); the input goes
// through the wave's LDS and transposing reads, one group ahead, and the waves'
// sums are added in LDS at the end.

constexpr int kGroup = 16;  // tokens of an MFMA (of fp16)
constexpr int kFew = 64;

struct Piece {
  int t0, t1;        // in perm
  long long group0;  // of the packed groups: those of pieces before it are fewer
  int index;
};
__device__ __forceinline__ Piece piece_of(const OuterArgs& a, int adapter, int split) {
  const int b0 = a.first ? a.first[adapter] : 0;
  const int b1 = a.first ? a.first[adapter + 1] : adapter == 0 ? a.n_tokens : 0;
  const int per = ((b1 - b0 + a.splits - 1) / a.splits + kGroup - 1) / kGroup * kGroup;
  Piece p;
  p.t0 = min(b1, b0 + split * per);
  p.t1 = min(b1, p.t0 + per);
  p.index = adapter * a.splits + split;
  p.group0 = p.t0 / kGroup + p.index;
  return p;
}

// the scale of a piece, from each token's largest; `all`: W floats of LDS
template <int W>
__device__ __forceinline__ void piece_scale(const OuterArgs& a, const Outer& m, const Piece& p, float* all, float& up, float& down) {
  float largest = 0.0f;
#pragma unroll 4
  for (int t = p.t0 + (int)threadIdx.x; t < p.t1; t += 64 * W) largest = fmaxf(largest, m.most[a.perm ? a.perm[t] : t]);
#pragma unroll
  for (int d = 1; d < 64; d <<= 1) largest = fmaxf(largest, __shfl_xor(largest, d));
  if ((threadIdx.x & 63) == 0) all[threadIdx.x >> 6] = largest;
  __syncthreads();
#pragma unroll
  for (int w = 0; w < W; ++w) largest = fmaxf(largest, all[w]);
  __syncthreads();
  pick_scale(largest, up, down);
}

// The places of the tokens t .. t + 7 of a piece that ends at t1; those past its
// end repeat its last (loads without a branch each are in flight together).
__device__ __forceinline__ void rows_of(const OuterArgs& a, int t, int t1, int (&at)[8]) {
#pragma unroll
  for (int e = 0; e < 8; ++e) at[e] = min(t + e, t1 - 1);
  if (a.perm) {
#pragma unroll
    for (int e = 0; e < 8; ++e) at[e] = a.perm[at[e]];
  }
}

template <int RB>  // 32 RB ranks
__global__ __launch_bounds__(kThreads) void pack_kernel(OuterArgs a) {
  __shared__ float all[kWaves];
  const int which = (int)blockIdx.z / a.count, adapter = (int)blockIdx.z % a.count;
  const Outer& m = a.m[which];
  const Piece p = piece_of(a, adapter, blockIdx.y);
  const int n = p.t1 - p.t0;
  if (n <= kFew) return;  // (what it would pack is not read)
  float up, down;
  piece_scale<kWaves>(a, m, p, all, up, down);
  if (threadIdx.x == 0 && blockIdx.x == 0) m.down[p.index] = down;
  // one lane's operand at a time
  const int groups = (n + kGroup - 1) / kGroup;
  for (int q = (int)blockIdx.x * kThreads + threadIdx.x; q < groups * RB * 64; q += (int)gridDim.x * kThreads) {
    const int lane = q & 63, block = (q >> 6) % RB, g = (q >> 6) / RB;
    const int j = 32 * block + (lane & 31);
    const int t = p.t0 + g * kGroup + 8 * (lane >> 5);
    int at[8];
    float v[8];
    half8 hi, lo;
    rows_of(a, t, p.t1, at);
#pragma unroll
    for (int e = 0; e < 8; ++e) v[e] = m.act[(uint32_t)at[e] * (uint32_t)a.rank + (uint32_t)min(j, a.rank - 1)];
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      _Float16 h, l;
      split2(t + e < p.t1 && j < a.rank ? v[e] * up : 0.0f, h, l);
      hi[e] = h;
      lo[e] = l;
    }
    half8* const to = reinterpret_cast<half8*>(m.packed) + ((p.group0 + g) * RB + block) * 128 + lane;
    to[0] = hi;
    to[64] = lo;
  }
}

// The waves of a SIMD that the form of few tokens, which needs more registers, must
// not cost the other.
constexpr int outer_occupancy(int rb, int w, int fb, bool direct) {
  return direct || w == 8 ? 1 : rb * fb == 8 ? 2 : rb == 2 ? 4 : 3;
}

template <int RB, int W, int FB, bool DIRECT>  // 32 RB ranks, W waves, 32 FB columns
__global__ __launch_bounds__(64 * W, outer_occupancy(RB, W, FB, DIRECT)) void outer_kernel(OuterArgs a) {
  constexpr int kRow = 64 * FB + 16;  // bytes of a token's columns in LDS, padded
  constexpr int kRowLanes = 4 * FB;   // lanes that load a token's columns
  constexpr int kRows = 64 / kRowLanes;
  constexpr int kRed = 4 * W * 2 * 16 * 64;
  constexpr int kIn = W * kGroup * kRow;
  static_assert(kFew <= W * kGroup, "few tokens are one group a wave");
  __shared__ __attribute__((aligned(16))) unsigned char lds[kRed > kIn ? kRed : kIn];
  const int lane = threadIdx.x & 63;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int which = (int)blockIdx.z / a.count, adapter = (int)blockIdx.z % a.count;
  const Outer& m = a.m[which];
  const int f0 = (int)blockIdx.x * 32 * FB;
  if (f0 >= m.width) return;
  const Piece piece = piece_of(a, adapter, blockIdx.y);

  float16v acc[RB][FB];
#pragma unroll
  for (int j = 0; j < RB; ++j)
#pragma unroll
    for (int i = 0; i < FB; ++i) acc[j][i] = float16v{};
  unsigned char* const mine = lds + wave * kGroup * kRow;
  const int col = f0 + 8 * (lane % kRowLanes);
  const int left = m.width - col;
  const half8* const packed = reinterpret_cast<const half8*>(m.packed) + piece.group0 * RB * 128 + lane;
  const int groups = (piece.t1 - piece.t0 + kGroup - 1) / kGroup;
  const half8 none = half8{0, 0, 0, 0, 0, 0, 0, 0};
  const bool few = piece.t1 - piece.t0 <= kFew;
  float up = 1.0f, down = 1.0f;
  if constexpr (DIRECT) {
    if (!few) piece_scale<W>(a, m, piece, reinterpret_cast<float*>(lds), up, down);
  }

  // a group's input and operands, requested a group ahead, its tokens' places
  // two ahead
  int at[FB];
  half8 in[FB], act[DIRECT ? 1 : 2 * RB];
  float raw[DIRECT ? RB : 1][8];
  auto places = [&](int g) __attribute__((always_inline)) {
#pragma unroll
    for (int p = 0; p < FB; ++p) {
      const int t = piece.t0 + g * kGroup + kRows * p + lane / kRowLanes;
      at[p] = t < piece.t1 ? (a.perm ? a.perm[t] : t) : -1;
    }
  };
  auto request_in = [&]() __attribute__((always_inline)) {
#pragma unroll
    for (int p = 0; p < FB; ++p) in[p] = none;
    if (!DIRECT && m.stream) {
#pragma unroll
      for (int p = 0; p < FB; ++p)
        if (at[p] >= 0 && left > 0) in[p] = load8_once(m.in + (size_t)at[p] * m.width + col, left);
    } else {
#pragma unroll
      for (int p = 0; p < FB; ++p)
        if (at[p] >= 0 && left > 0) in[p] = load8_inside(m.in + (size_t)at[p] * m.width + col, left);
    }
  };
  auto keep_in = [&]() __attribute__((always_inline)) {
#pragma unroll
    for (int p = 0; p < FB; ++p)
      *reinterpret_cast<half8*>(mine + (kRows * p + lane / kRowLanes) * kRow + 16 * (lane % kRowLanes)) = in[p];
  };
  // the activations of ranks 32 j + lane mod 32 and of the lane's eight tokens
  auto load_raw = [&](int g, auto& to) __attribute__((always_inline)) {
    int from[8];
    rows_of(a, piece.t0 + g * kGroup + 8 * (lane >> 5), piece.t1, from);
#pragma unroll
    for (int e = 0; e < 8; ++e)
#pragma unroll
      for (int j = 0; j < RB; ++j) {
        const uint32_t bytes = 4u * ((uint32_t)from[e] * (uint32_t)a.rank + (uint32_t)min(32 * j + (lane & 31), a.rank - 1));
        to[j][e] = *reinterpret_cast<const float*>(reinterpret_cast<const char*>(m.act) + bytes);
      }
  };
  auto there = [&](int g, int j, int e) __attribute__((always_inline)) {
    return piece.t0 + g * kGroup + 8 * (lane >> 5) + e < piece.t1 && 32 * j + (lane & 31) < a.rank;
  };
  auto request = [&](int g) __attribute__((always_inline)) {
    request_in();
    if constexpr (DIRECT) {
      load_raw(g, raw);
    } else {
#pragma unroll
      for (int j = 0; j < 2 * RB; ++j) act[j] = packed[(size_t)g * RB * 128 + 64 * j];
    }
  };
  int g = wave;
  if (few && g < groups) {
    float x[RB][8];
    places(g);
    request_in();
    load_raw(g, x);
    keep_in();
    wave_fence();
#pragma unroll
    for (int j = 0; j < RB; ++j)
#pragma unroll
      for (int e = 0; e < 8; ++e) x[j][e] = there(g, j, e) ? x[j][e] : 0.0f;
#pragma unroll
    for (int i = 0; i < FB; ++i) {
      const half8 v = read_transposed(mine, kRow, 0, 32 * i);
#pragma unroll
      for (int e = 0; e < 8; ++e) {
#pragma unroll
        for (int j = 0; j < RB; ++j) acc[j][i] = __builtin_amdgcn_mfma_f32_32x32x2f32(x[j][e], (float)v[e], acc[j][i], 0, 0, 0);
      }
      __builtin_amdgcn_sched_barrier(0);
    }
  }
  if (few) g = groups;
  if (g < groups) {
    places(g);
    request(g);
    places(g + W);
  }
  for (; g < groups; g += W) {
    half8 now[2 * RB];
    keep_in();
    if constexpr (DIRECT) {
#pragma unroll
      for (int j = 0; j < RB; ++j)
#pragma unroll
        for (int e = 0; e < 8; ++e) {
          _Float16 hi, lo;
          split2(there(g, j, e) ? raw[j][e] * up : 0.0f, hi, lo);
          now[2 * j][e] = hi;
          now[2 * j + 1][e] = lo;
        }
    } else {
#pragma unroll
      for (int j = 0; j < 2 * RB; ++j) now[j] = act[j];
    }
    if (g + W < groups) {
      request(g + W);
      places(g + 2 * W);
    }
    wave_fence();
#pragma unroll
    for (int i = 0; i < FB; ++i) {
      const half8 v = read_transposed(mine, kRow, 0, 32 * i);
#pragma unroll
      for (int j = 0; j < RB; ++j) {
        acc[j][i] = __builtin_amdgcn_mfma_f32_32x32x16_f16(now[2 * j], v, acc[j][i], 0, 0, 0);
        acc[j][i] = __builtin_amdgcn_mfma_f32_32x32x16_f16(now[2 * j + 1], v, acc[j][i], 0, 0, 0);
      }
    }
    wave_fence();
  }

  if constexpr (!DIRECT) down = few ? 1.0f : m.down[piece.index];
  const float by = down * a.scale[adapter];
  float* const red = reinterpret_cast<float*>(lds);  // [wave][two column blocks][register][lane]
  float* const out = m.out + ((size_t)blockIdx.y * a.count + adapter) * a.rank * m.width;
#pragma unroll
  for (int j = 0; j < RB; ++j)
#pragma unroll
    for (int i0 = 0; i0 < FB; i0 += 2) {
      __syncthreads();
#pragma unroll
      for (int i = 0; i < 2; ++i)
#pragma unroll
        for (int e = 0; e < 16; ++e) red[((wave * 2 + i) * 16 + e) * 64 + lane] = acc[j][i0 + i][e];
      __syncthreads();
      // a wave adds its share of the 32 (block, register) pairs
#pragma unroll
      for (int q = 0; q < 32 / W; ++q) {
        const int i = q & 1, e = 16 / W * wave + (q >> 1);
        float sum = red[(i * 16 + e) * 64 + lane];
#pragma unroll
        for (int w = 1; w < W; ++w) sum += red[((w * 2 + i) * 16 + e) * 64 + lane];
        const int r = 32 * j + 8 * (e >> 2) + 4 * (lane >> 5) + (e & 3);
        const int f = f0 + 32 * (i0 + i) + (lane & 31);
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
                                                            Tile* tiles, int max_tiles, int per_tile) {
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
    n_tiles += (sum + per_tile - 1) / per_tile;
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
    const int of = (end - base[b] + per_tile - 1) / per_tile;
    for (int q = lane; q < of; q += 64)
      tiles[tile0[b] + q] = Tile{b < count ? b : -1, base[b] + q * per_tile, min(per_tile, end - base[b] - q * per_tile), 0};
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

using namespace spdp;

constexpr int kLdsPlain = 48 * 1024;  // dynamic LDS that a launch may have without asking

// The ranges of the width that shrink_kernel's workgroups take: one workgroup
// per CU, at least four steps each (one per wave), at most eight ranges, for
// expand_kernel's workgroups all add them (whole passes of rank 64 with 2 / 4 / 8 /
// 16 ranges: 4096 tokens, 13824 to 5120, 89 / 66 / 70 / 83 us; 1000, 11008 to 4096, 40 /
// 27 / 22 / 26).
struct Ranges {
  int per, splits;
};
Ranges shrink_ranges(int64_t width, long long tiles, int banks, int cus) {
  const int steps = (int)((width + kStep - 1) / kStep);
  const int most = std::max(1, std::min(8, steps / 4));
  const int want = (int)std::min<long long>(most, (cus + tiles * banks - 1) / (tiles * banks));
  const int per = (steps + want - 1) / want;
  return {per, (steps + per - 1) / per};
}

// The workgroups of outer_kernel without a split, the pieces that an adapter's
// tokens are split into, and the waves of a workgroup: pieces of many tokens, four
// workgroups per CU (a CU holds five, four or two at up to 32, 64 and 128 ranks);
// unsplit, eight waves where there are fewer than two workgroups per CU. Whole backward passes, us, unsplit of
// four waves / of eight / split: 4096 tokens, 13824 x 5120, rank 64 143 / 144 /
// 129; 2048, 4096 x 11008, rank 16 62 / 53 / 54; 4000 of 8 adapters, 8192 x 8192,
// rank 8 107 / 111 / 108.
//
// Much input and ranks up to 64: 128 columns, which read the packed activations
// half as often (they come from L2, twice the input's bytes at rank 64 and 64
// columns), and the pieces that fill the two workgroups that a CU holds best
// (4096 tokens, 13824 x 5120, rank 64 129 -> 120 us; 16384, 4096 x 4096, rank 16
// 167 -> 155; 3000, 11008 x 4096, rank 32 would take 77 for 74).
long long outer_wgs(const spdp_adapters_t* m, int cols) {
  return ((m->rows + cols - 1) / cols + (m->cols + cols - 1) / cols) * m->count;
}
bool outer_wide(const spdp_adapters_t* m, long long n_tokens) {
  return m->rank <= 64 && n_tokens / m->count > 2500 && n_tokens * (m->rows + m->cols) > 70000000;
}
int outer_splits(const spdp_adapters_t* m, long long n_tokens, int cus) {
  if (n_tokens / m->count <= 2500) return 1;
  if (!outer_wide(m, n_tokens)) return (int)std::min<long long>(16, std::max<long long>(1, 4 * cus / outer_wgs(m, kCols)));
  int best = 1;
  float most = 0.0f;
  for (int s = 1; s <= 8; ++s) {
    const long long wgs = outer_wgs(m, 2 * kCols) * s, slots = 2ll * cus;
    const float fill = (float)wgs / (float)((wgs + slots - 1) / slots * slots) - 0.05f * (float)s;
    if (fill > most) {
      most = fill;
      best = s;
    }
  }
  return best;
}
// and their packed activations: the groups of 16 tokens, one more per piece
size_t packed_bytes(const spdp_adapters_t* m, long long n_tokens, int splits) {
  const size_t block = m->rank <= 32 ? 1 : m->rank <= 64 ? 2 : 4;
  return aligned(((size_t)n_tokens / kGroup + (size_t)m->count * splits + 1) * block * 2 * 64 * 16);
}

// What the sort writes, and where, and the launch's tiles.
struct SortPlan {
  bool sorted;
  int tile;         // tokens of a tile
  long long tiles;  // of the grid
  size_t bytes;     // perm, first, tiles
};
SortPlan plan_sort(long long n_tokens, int count, int banks, bool ids, bool always, int cus) {
  SortPlan p;
  p.sorted = ids && (always || n_tokens > kSmall);
  // larger tiles read the factors less often; smaller ones make more workgroups
  // where there are few tokens, and waste less where an adapter has few
  const long long own = ids ? n_tokens / std::min<long long>(count, n_tokens) : n_tokens;
  p.tile = own >= 128 && n_tokens * banks >= 8ll * cus ? 64 : own >= 24 ? 32 : 16;
  p.tiles = !ids ? (n_tokens + p.tile - 1) / p.tile
            : p.sorted ? n_tokens / p.tile + std::min<long long>(count + 1, n_tokens) + 1
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

// fp32 of the rank activations' partial sums
size_t part_bytes(long long n_tokens, int rank, int splits) { return aligned((size_t)splits * n_tokens * rank * 4); }

int sort_tokens(const int32_t* ids, long long n, int count, const SortPlan& p, unsigned char* ws, Tokens* t, int** first,
                hipStream_t st) {
  int* const perm = reinterpret_cast<int*>(ws);
  *first = reinterpret_cast<int*>(ws + aligned((size_t)n * 4));
  Tile* const tiles = reinterpret_cast<Tile*>(ws + aligned((size_t)n * 4) + aligned((size_t)(count + 2) * 4));
  const int lds = (kSortWaves + 2) * (count + 1) * 4;
  if (lds > kLdsPlain) {
    const hipError_t e =
        hipFuncSetAttribute(reinterpret_cast<const void*>(sort_kernel), hipFuncAttributeMaxDynamicSharedMemorySize, lds);
    if (e != hipSuccess) return hip_fail(e, "hipFuncSetAttribute");
  }
  hipLaunchKernelGGL(sort_kernel, dim3(1), dim3(kSortThreads), lds, st, ids, (int)n, count, perm, *first, tiles,
                     (int)p.tiles, p.tile);
  const hipError_t e = hipGetLastError();
  if (e != hipSuccess) return hip_fail(e, "kernel launch");
  t->perm = perm;
  t->tiles = tiles;
  return SPDP_OK;
}

template <int RB, int T>
hipError_t launch_shrink_form(const ShrinkArgs& a, dim3 grid, hipStream_t st) {
  // eight waves where a wave's registers let two of them share a SIMD and it loads
  // one step at a time (2048 tokens, rank 32, 28672 wide: the backward pass 133 ->
  // 116 us); smaller forms load two steps at a time and would wait longer for their
  // sums (32 tokens, rank 16, 4096 x 4096: 8.4 -> 9.4)
  constexpr int W = RB + T / 16 == 6 ? 2 * kWaves : kWaves;
  const int lds = W * T * 16 * RB * 4;
  if (lds > kLdsPlain) {
    const hipError_t e = hipFuncSetAttribute(reinterpret_cast<const void*>(shrink_kernel<RB, T, W>),
                                             hipFuncAttributeMaxDynamicSharedMemorySize, lds);
    if (e != hipSuccess) return e;
  }
  hipLaunchKernelGGL((shrink_kernel<RB, T, W>), grid, dim3(64 * W), lds, st, a);
  return hipGetLastError();
}
template <int RB>
hipError_t launch_shrink_rb(const ShrinkArgs& a, int tile, dim3 grid, hipStream_t st) {
  return tile == 16   ? launch_shrink_form<RB, 16>(a, grid, st)
         : tile == 32 ? launch_shrink_form<RB, 32>(a, grid, st)
                      : launch_shrink_form<RB, 64>(a, grid, st);
}
hipError_t launch_shrink(const ShrinkArgs& a, int tile, dim3 grid, hipStream_t st) {
  if (a.rank <= 16) return launch_shrink_rb<1>(a, tile, grid, st);
  if (a.rank <= 32) return launch_shrink_rb<2>(a, tile, grid, st);
  if (a.rank <= 64) return launch_shrink_rb<4>(a, tile, grid, st);
  return launch_shrink_rb<8>(a, tile, grid, st);
}

// Outputs, or an input, of all tokens that are larger than the L2 caches (4 MB on
// each of 8 dies). The outer products' inputs go past the caches, too, for nothing
// reads them afterwards: backward passes of 4096 tokens, rank 64, 13824 x 5120,
// 118.6 -> 112.3 us; 1000 of rank 64, 4096 x 11008, which fit, would take 43.1 for 41.
bool streams(long long n_tokens, int64_t width) { return n_tokens * width * 2 > 32ll << 20; }

template <int RB, int T, bool FUSED, bool ONCE>
hipError_t launch_expand_form(const ExpandArgs& a, dim3 grid, hipStream_t st) {
  constexpr int W = FUSED ? kFusedWaves : kWaves;
  const int lds = ExpandCfg<RB, T, W>::kLds;
  if (lds > kLdsPlain) {
    const hipError_t e = hipFuncSetAttribute(reinterpret_cast<const void*>(expand_kernel<RB, T, FUSED, ONCE>),
                                             hipFuncAttributeMaxDynamicSharedMemorySize, lds);
    if (e != hipSuccess) return e;
  }
  hipLaunchKernelGGL((expand_kernel<RB, T, FUSED, ONCE>), grid, dim3(64 * W), lds, st, a);
  return hipGetLastError();
}
template <int RB>
hipError_t launch_expand_rb(const ExpandArgs& a, int tile, bool once, dim3 grid, hipStream_t st) {
  if (once)
    return tile == 16 ? launch_expand_form<RB, 16, false, true>(a, grid, st) : launch_expand_form<RB, 32, false, true>(a, grid, st);
  return tile == 16 ? launch_expand_form<RB, 16, false, false>(a, grid, st) : launch_expand_form<RB, 32, false, false>(a, grid, st);
}
template <int RB>
hipError_t launch_fused_rb(const ExpandArgs& a, int tile, dim3 grid, hipStream_t st) {
  return tile == 16 ? launch_expand_form<RB, 16, true, false>(a, grid, st) : launch_expand_form<RB, 32, true, false>(a, grid, st);
}
hipError_t launch_expand(ExpandArgs& a, int banks, const SortPlan& p, bool fused, int cus, hipStream_t st) {
  // (with 64 tokens a workgroup of expand_kernel was slower: 65 us for 56 of 2048
  // tokens of rank 32, 28672 wide, 33 for 30 of 4096 of rank 64, 5120 wide)
  a.subs = p.tile > 32 ? p.tile / 32 : 1;
  const long long tiles = p.tiles * a.subs;
  int widest = 0;
  int64_t all = 0;
  for (int i = 0; i < banks; ++i) {
    widest = std::max(widest, a.m[i].width);
    all += a.m[i].width;
  }
  const int block = kCols * (fused ? kFusedWaves : kWaves);
  const int blocks = (widest + block - 1) / block;
  // a workgroup keeps its tokens' activations for several blocks where that
  // leaves the three workgroups that a CU holds (whole passes over 2048 tokens of
  // rank 32, 28672 wide, with 2 / 3 / 5 / 8 blocks: 79 / 80 / 78 / 90 us)
  const long long fill = (fused ? 1ll : 3ll) * cus;
  a.blocks = (int)std::max<long long>(1, std::min<long long>(5, (blocks * tiles * banks + fill - 1) / fill));
  const dim3 grid((unsigned)((blocks + a.blocks - 1) / a.blocks), (unsigned)tiles, (unsigned)banks);
  // (the fused form's outputs are never so large)
  const bool once = streams(a.t.n_tokens, all);
  if (fused)
    return a.rank <= 16   ? launch_fused_rb<1>(a, p.tile, grid, st)
           : a.rank <= 32 ? launch_fused_rb<2>(a, p.tile, grid, st)
                          : launch_fused_rb<4>(a, p.tile, grid, st);
  if (a.rank <= 16) return launch_expand_rb<1>(a, p.tile, once, grid, st);
  if (a.rank <= 32) return launch_expand_rb<2>(a, p.tile, once, grid, st);
  if (a.rank <= 64) return launch_expand_rb<4>(a, p.tile, once, grid, st);
  return launch_expand_rb<8>(a, p.tile, once, grid, st);
}

template <int RB, bool DIRECT>
hipError_t launch_outer_form(const OuterArgs& a, int widest, hipStream_t st) {
  const int cols = a.wide ? 2 * kCols : kCols;
  const dim3 grid((unsigned)((widest + cols - 1) / cols), (unsigned)a.splits, (unsigned)(2 * a.count));
  if (a.wide) {
    if constexpr (RB <= 2 && !DIRECT) hipLaunchKernelGGL((outer_kernel<RB, 4, 4, false>), grid, dim3(256), 0, st, a);
  } else if (a.waves == 4) {
    hipLaunchKernelGGL((outer_kernel<RB, 4, 2, DIRECT>), grid, dim3(256), 0, st, a);
  } else if constexpr (!DIRECT || RB <= 2) {
    hipLaunchKernelGGL((outer_kernel<RB, 8, 2, DIRECT>), grid, dim3(512), 0, st, a);
  }
  return hipGetLastError();
}
template <int RB>
hipError_t launch_outer_rb(const OuterArgs& a, int widest, hipStream_t st) {
  if (a.packed == 0) return launch_outer_form<RB, true>(a, widest, st);
  // four workgroups a piece, or up to 64 where there are few pieces
  const unsigned share = (unsigned)std::max(4, std::min(64, 256 / (a.splits * a.count)));
  hipLaunchKernelGGL(pack_kernel<RB>, dim3(share, (unsigned)a.splits, (unsigned)(2 * a.count)), dim3(kThreads), 0, st, a);
  const hipError_t e = hipGetLastError();
  return e != hipSuccess ? e : launch_outer_form<RB, false>(a, widest, st);
}
hipError_t launch_outer(const OuterArgs& a, int widest, hipStream_t st) {
  if (a.rank <= 32) return launch_outer_rb<1>(a, widest, st);
  if (a.rank <= 64) return launch_outer_rb<2>(a, widest, st);
  return launch_outer_rb<4>(a, widest, st);
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
  bool fused;
  size_t bytes;
};
void plan_adapt(const spdp_adapters_t* banks, int n_banks, long long n_tokens, bool ids, int cus, AdaptPlan* p) {
  std::memset(p, 0, sizeof(*p));
  p->sort = plan_sort(n_tokens, banks[0].count, n_banks, ids, false, cus);
  p->bytes = p->sort.bytes;
  p->splits = 1;
  // The fused form, where a workgroup's own pass over the first factor (at 16,
  // 32 or 64 ranks) is short and the workgroups that make it are few. Two
  // launches -> fused, us per pass from a graph: one token of rank 8, 1024 wide, 6.5
  // -> 4.5; 24 of 5 adapters of rank 12, 5003 x 3080, 7.6 -> 7.7, a launch less for
  // the host; one of rank 16, 4096 wide, 6.2 -> 8.2; 333 of 4 adapters of rank 16,
  // 1024 wide (and the sort) 13.4 -> 11.8, 4096 wide 14.2 -> 21.2.
  long long wgs = 0;
  p->fused = p->sort.tile <= 32 && banks[0].rank <= 64;
  for (int i = 0; i < n_banks; ++i) {
    p->fused = p->fused && (banks[i].rank + 15) / 16 * 16 * banks[i].cols <= (p->sort.tile == 16 ? 50000 : 20000);
    wgs += p->sort.tiles * ((banks[i].rows + kCols * kFusedWaves - 1) / (kCols * kFusedWaves));
  }
  p->fused = p->fused && 2 * wgs <= 3 * cus;
  for (int i = 0; i < n_banks && !p->fused; ++i) {
    p->r[i] = shrink_ranges(banks[i].cols, p->sort.tiles, n_banks, cus);
    p->splits = std::max(p->splits, p->r[i].splits);
    p->bytes += part_bytes(n_tokens, banks[i].rank, p->r[i].splits);
  }
}

struct GradPlan {
  SortPlan sort;
  Ranges r;
  int splits;
  size_t part, u, outer[2], packed, down, most, bytes;
};
void plan_grad(const spdp_adapters_t* m, long long n_tokens, bool ids, int cus, GradPlan* p) {
  p->sort = plan_sort(n_tokens, m->count, 1, ids, true, cus);
  p->r = shrink_ranges(m->rows, p->sort.tiles, 1, cus);
  p->splits = outer_splits(m, n_tokens, cus);
  p->part = part_bytes(n_tokens, m->rank, p->r.splits);
  p->u = part_bytes(n_tokens, m->rank, 1);
  const size_t each = (size_t)p->splits * m->count * m->rank * 4;
  p->outer[0] = p->splits > 1 ? aligned(each * m->cols) : 0;
  p->outer[1] = p->splits > 1 ? aligned(each * m->rows) : 0;
  // (backward passes, 4096 x 4096, packed / direct: 200 tokens of rank 16 16.8 / 15.0
  // us, 400 of four adapters 24.9 / 22.8, 800 of eight of rank 64 41.0 / 42.9)
  const bool packed = n_tokens > 512;
  p->packed = packed ? packed_bytes(m, n_tokens, p->splits) : 0;
  p->down = packed ? aligned((size_t)m->count * p->splits * 4) : 0;
  p->most = aligned((size_t)n_tokens * 8);
  p->bytes = p->sort.bytes + p->part + p->u + p->outer[0] + p->outer[1] + 2 * (p->packed + p->down) + p->most;
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
    if (overlap(Y[i], out, ids, n * 4) || (H && overlap(H[i], kept, ids, n * 4)))
      return fail(SPDP_ERR_INVALID_ARG, "an output overlaps the ids");
    for (int j = 0; j < n_banks; ++j) {
      const size_t fac = (size_t)banks[j].count * banks[j].rank, other = n * banks[j].rows * 2;
      const Array in[] = {{X[j], n * banks[j].cols * 2},
                          {banks[j].a, fac * banks[j].cols * 2},
                          {banks[j].b, fac * banks[j].rows * 2},
                          {banks[j].scale, (size_t)banks[j].count * 4}};
      for (const Array& v : in) {
        if (overlap(Y[i], out, v.p, v.bytes)) return fail(SPDP_ERR_INVALID_ARG, "an output overlaps an input");
        if (H && overlap(H[i], kept, v.p, v.bytes)) return fail(SPDP_ERR_INVALID_ARG, "H overlaps another array");
      }
      if (overlap(Y[i], out, base[j], other) && !(i == j && Y[i] == base[j]))
        return fail(SPDP_ERR_INVALID_ARG, "an output overlaps a base other than its own as a whole");
      if (i != j && overlap(Y[i], out, Y[j], other)) return fail(SPDP_ERR_INVALID_ARG, "outputs overlap");
      if (H && (overlap(H[i], kept, base[j], other) || overlap(H[i], kept, Y[j], other) ||
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
    if (!p.fused) ws += part_bytes(n_tokens, b.rank, p.r[i].splits);
    sa.m[i] = Shrink{X[i], b.a, part, (int)b.cols, p.r[i].per};
    ea.m[i] = Expand{part, b.b, b.scale, base[i], Y[i], H ? H[i] : nullptr, nullptr, nullptr, X[i], b.a,
                       (int)b.rows, p.fused ? 1 : p.r[i].splits, (int)b.cols};
  }
  hipError_t e = hipSuccess;
  if (!p.fused) e = launch_shrink(sa, p.sort.tile, dim3((unsigned)p.sort.tiles, (unsigned)p.splits, (unsigned)n_banks), s);
  if (e == hipSuccess) e = launch_expand(ea, n_banks, p.sort, p.fused, cus, s);
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
  const Array in[] = {{X, n * bank->cols * 2}, {H, n * bank->rank * 4}, {dY, n * bank->rows * 2}, {base, n * bank->cols * 2},
                      {bank->a, fac * bank->cols * 2}, {bank->b, fac * bank->rows * 2}, {bank->scale, (size_t)bank->count * 4},
                      {ids, n * 4}};
  const Array out[] = {{dX, n * bank->cols * 2}, {dA, fac * bank->cols * 4}, {dB, fac * bank->rows * 4}};
  for (const Array& o : out) {
    for (const Array& i : in)
      if (overlap(o.p, o.bytes, i.p, i.bytes) && !(&o == &out[0] && &i == &in[3] && i.p == o.p))
        return fail(SPDP_ERR_INVALID_ARG, "an output overlaps an input (dX may be its base as a whole)");
    for (const Array& q : out)
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
  unsigned char* const packed = ws + p.part + p.u + p.outer[0] + p.outer[1];
  float* const down = reinterpret_cast<float*>(packed + 2 * p.packed);
  float* const most = reinterpret_cast<float*>(packed + 2 * (p.packed + p.down));
  ShrinkArgs sa;
  ExpandArgs ea;
  OuterArgs oa;
  std::memset(&sa, 0, sizeof(sa));
  std::memset(&ea, 0, sizeof(ea));
  std::memset(&oa, 0, sizeof(oa));
  sa.t = ea.t = t;
  sa.rank = ea.rank = oa.rank = bank->rank;
  sa.m[0] = Shrink{dY, bank->b, part, (int)bank->rows, p.r.per};
  ea.m[0] = Expand{part, bank->a, bank->scale, base, dX, u, most, H, nullptr, nullptr, (int)bank->cols, p.r.splits, 0};
  hipError_t e = launch_shrink(sa, p.sort.tile, dim3((unsigned)p.sort.tiles, (unsigned)p.r.splits, 1), s);
  if (e == hipSuccess) e = launch_expand(ea, 1, p.sort, false, cus, s);
  if (e != hipSuccess) return hip_fail(e, "kernel launch");
  const bool split = p.splits > 1;
  oa.m[0] = Outer{u, X, split ? pa : dA, most, packed, down, (int)bank->cols, streams(n_tokens, bank->cols)};
  oa.m[1] = Outer{H, dY, split ? pb : dB, most + n_tokens, packed + p.packed,
                  down + p.down / 4, (int)bank->rows, streams(n_tokens, bank->rows)};
  oa.scale = bank->scale;
  oa.perm = t.perm;
  oa.first = first;
  oa.n_tokens = (int)n_tokens;
  oa.count = bank->count;
  oa.splits = p.splits;
  oa.wide = outer_wide(bank, n_tokens);
  oa.packed = p.packed > 0;
  // (the direct form of more than 64 ranks spills registers with eight: 39.3 us of 64
  // tokens of four adapters, rank 128, 4096 x 4096, with either)
  oa.waves = !split && outer_wgs(bank, kCols) < 2 * cus && (oa.packed || bank->rank <= 64) ? 8 : 4;
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
