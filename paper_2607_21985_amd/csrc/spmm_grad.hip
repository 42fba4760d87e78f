// Gradient of the prefill product with respect to its input: dX = dY W_sp for
// N tokens, on the encoded arrays of the forward product (nothing dense or
// transposed is kept). The contraction runs over the matrix rows, along which
// a column's values are stored: a lane that owns a column walks down its
// values, and eight rows of it are an MFMA operand as they come.
//
//   * grad_kernel, for handles with word records: a wave owns 32 columns and
//     32 TB tokens, and expands from LDS into operand registers (described at
//     the kernel);
//   * grad_plain_kernel, for the others.
//
// Measured (whole calls among others), 13824 x 5120 at 70 % sparsity, 2048 tokens:
// 324 to 331 us, 890 TFLOP/s of the dense product that the matrix cores execute; they
// are busy half of the cycles, LDS and vector issue nearly as long, and the power
// limit holds the clock (283 us on a dY of zeros; under a tracer 346 to 374 and 26 for
// the second launch). 4096 x 4096 at 50 %, 256 tokens: 26 us, bound by vector issue
// and the second launch.

#include <hip/hip_fp16.h>
#include <hip/hip_runtime.h>

#include <algorithm>
#include <cstdlib>
#include <cstring>

#include "calls.h"
#include "lanes.h"

namespace {

using namespace spdp_dev;

constexpr int kTM = 256;  // rows of a stripe: four words
constexpr int kThreads = 256;

struct GradArgs {
  const uint32_t* tile_offset;
  const uint32_t* col_info;
  const uint64_t* bitmap;
  const unsigned char* rec;
  const uint32_t* chunk_off;
  const uint16_t* values;
  const uint16_t* dy;  // [n_tokens][rows]
  uint16_t* dx;        // [n_tokens][cols]
  float* part;         // [splits][n_tokens][cols] fp32 with more than one split
  long long n_tokens;
  int rows, cols;
  int tk_log2, n_colblocks;
  int n_stripes;
  int per;             // stripes of a split
  int chunks;
  int run;             // LDS bytes of a stripe's values
};

// 32 tokens x 32 columns: register e of lane l holds token 8 (e / 4) + 4 (l / 32)
// + e mod 4 and column l mod 32, so that a store writes 64 bytes of two tokens
__device__ __forceinline__ void store_sums(const GradArgs& a, const float16v& acc, long long n0, int col) {
  if (col >= a.cols) return;
  float* const part = gridDim.z > 1 ? a.part + (size_t)blockIdx.z * (size_t)a.n_tokens * (size_t)a.cols : nullptr;
#pragma unroll
  for (int e = 0; e < 16; ++e) {
    const long long n = n0 + 8 * (e >> 2) + 4 * ((threadIdx.x & 63) >> 5) + (e & 3);
    if (n >= a.n_tokens) continue;
    if (part)
      __builtin_nontemporal_store(acc[e], part + n * (long long)a.cols + col);
    else
      a.dx[n * (long long)a.cols + col] = __half_as_ushort(__float2half_rn(acc[e]));
  }
}

// The plain form: 64 columns x 128 tokens, a step of one 64-row word. Lanes are
// rows: each wave puts 16 columns into the LDS tile, column by column.
constexpr int kPlainRow = 144;  // bytes of a column's 64 rows, padded

__global__ __launch_bounds__(kThreads) void grad_plain_kernel(GradArgs a) {
  __shared__ __attribute__((aligned(16))) unsigned char tile[64 * kPlainRow];
  const int lane = threadIdx.x & 63;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int k0 = (int)blockIdx.x * 64;
  const long long n0 = (long long)blockIdx.y * 128 + 32 * wave;
  const long long tok = min(n0 + (lane & 31), a.n_tokens - 1);
  const uint16_t* const dy = a.dy + tok * (long long)a.rows;
  const int tk = 1 << a.tk_log2;
  float16v acc[2] = {float16v{}, float16v{}};
  const int r1 = min(a.n_stripes, ((int)blockIdx.z + 1) * a.per);
  for (int r = (int)blockIdx.z * a.per; r < r1; ++r) {
    for (int v = 0; v < 4; ++v) {
      if (r * kTM + 64 * v >= a.rows) break;
      __syncthreads();
      for (int c = 0; c < 16; ++c) {
        const int k = k0 + 16 * wave + c;
        uint16_t h = 0;
        if (k < a.cols) {
          const size_t g = (size_t)r * a.n_colblocks + (k >> a.tk_log2);
          const size_t at = g * tk + (k & (tk - 1));
          uint32_t base = a.tile_offset[g] + (a.col_info[at] >> 16);
          for (int u = 0; u < v; ++u) base += (uint32_t)__popcll(a.bitmap[at * 4 + u]);
          const uint64_t word = a.bitmap[at * 4 + v];
          if (word >> lane & 1) h = a.values[base + (uint32_t)__popcll(word & ((1ull << lane) - 1))];
        }
        *reinterpret_cast<uint16_t*>(tile + (16 * wave + c) * kPlainRow + 2 * lane) = h;
      }
      __syncthreads();
#pragma unroll
      for (int s = 0; s < 4; ++s) {
        const int m = r * kTM + 64 * v + 16 * s + 8 * (lane >> 5);
        const half8 x = m < a.rows ? load8_inside(dy + m, a.rows - m) : half8{0, 0, 0, 0, 0, 0, 0, 0};
#pragma unroll
        for (int i = 0; i < 2; ++i) {
          const half8 w = *reinterpret_cast<const half8*>(tile + (32 * i + (lane & 31)) * kPlainRow + 32 * s + 16 * (lane >> 5));
          acc[i] = __builtin_amdgcn_mfma_f32_32x32x16_f16(x, w, acc[i], 0, 0, 0);
        }
      }
    }
  }
#pragma unroll
  for (int i = 0; i < 2; ++i) store_sums(a, acc[i], n0, k0 + 32 * i + (lane & 31));
}

// ---------------------------------------------------------------------------
// The form for handles with word records. CG TG waves own 32 CG columns (CG / 2
// chunks) and 32 TB TG tokens, each wave 32 columns and 32 TB tokens; lane l has
// column l mod 32 and, of each stripe, the rows 128 (l / 32) .. + 127, whose
// values it walks down. Per four rows it puts the next values (as many as the
// four bits of the bitmap have ones) into their places with two byte
// permutations, whose selectors a table of 16 entries holds. Eight rows are an
// operand of v_mfma_f32_32x32x16_f16; the tokens' operands come from LDS in the
// same order of rows. The values are read as aligned 8-byte words, of which the
// last one is kept, and shifted in registers: a wave's 64 reads of 8 bytes take
// 6 cycles where all are aligned, 65 where they are not.
//
// A step is 8 rows of both halves of the lanes; a quarter of a stripe has four.
// During the MFMAs of a step the next one's operands are built and read, across
// quarters, too. Values (per stripe one contiguous run) arrive by DMA in three
// parts during the stripe before, a quarter's 64 rows of dY one quarter ahead,
// 16-byte piece p of token t at place p ^ (t / 2 mod 8). The one barrier per
// quarter stands where all of the quarter's operands have been read, two or four
// MFMAs before its end: what is requested behind it may overwrite them.

template <int TB, int CG, int TG>
struct GradCfg {
  static constexpr int kWaves = CG * TG;
  static constexpr int kTokens = 32 * TB * TG;
  static constexpr int kDyBytes = kTokens * 128;
  static int lds(int run) { return 2 * run + 2 * kDyBytes + 256; }
};

typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));

// Where a lane is in its column: the aligned 8 bytes of LDS that hold its next
// value, and the 8 behind them.
struct Window {
  u32x2 a, b;
  uint32_t at;
};
// Four rows of a column, requested: the 8 bytes behind those that hold the first
// value, and the selectors for the rows' bits.
struct Quad {
  u32x2 behind, sel;
  uint32_t p;
  __device__ __forceinline__ void read(uint32_t at, uint32_t selectors_at) {
    typedef const __attribute__((address_space(3))) u32x2* lds8;
    p = at;
    behind = *(lds8)(uintptr_t)((at & ~7u) + 8u);
    sel = *(lds8)(uintptr_t)selectors_at;
  }
  // the rows' fp16, 0 where the bit is clear; moves the window on (four rows
  // have at most 8 bytes of values, so by one word at most)
  __device__ __forceinline__ u32x2 rows(Window& w) const {
    const bool next = (p & ~7u) != w.at;
    w.a = next ? w.b : w.a;
    w.b = behind;
    w.at = p & ~7u;
    const bool up = p & 4u;
    const uint32_t x0 = up ? w.a[1] : w.a[0], x1 = up ? w.b[0] : w.a[1], x2 = up ? w.b[1] : w.b[0];
    const uint32_t lo = __builtin_amdgcn_alignbyte(x1, x0, p), hi = __builtin_amdgcn_alignbyte(x2, x1, p);
    return u32x2{__builtin_amdgcn_perm(hi, lo, sel[0]), __builtin_amdgcn_perm(hi, lo, sel[1])};
  }
};

// selectors of the two dwords of four rows with bitmap bits `b`
__device__ __forceinline__ u32x2 selectors(uint32_t b) {
  u32x2 s;
  uint32_t rank = 0;
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const uint32_t half = (b >> i & 1) ? 0x0100u + 0x0202u * rank : 0x0C0Cu;
    rank += b >> i & 1;
    s[i / 2] = (i & 1) ? s[i / 2] | half << 16 : half;
  }
  return s;
}

// DYV: dY rows are 16-byte aligned (else they are read at any address)
template <int TB, int CG, int TG, bool DYV>
__global__ __launch_bounds__(64 * CG * TG) void grad_kernel(GradArgs a) {
  using C = GradCfg<TB, CG, TG>;
  constexpr int W = C::kWaves;
  extern __shared__ __attribute__((aligned(1024))) unsigned char lds[];
  const int lane = threadIdx.x & 63;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int cg = wave % CG, tg = wave / CG;
  const int half = lane >> 5;
  const long long nb0 = (long long)blockIdx.y * C::kTokens;
  const int last_tok = (int)min(a.n_tokens - nb0, (long long)C::kTokens) - 1;
  const int chunk0 = CG / 2 * (int)blockIdx.x;
  const int chunk1 = min(chunk0 + CG / 2, a.chunks);
  const bool on = chunk0 + (cg >> 1) < chunk1;  // the last workgroup's chunks may be fewer
  const int chunk = on ? chunk0 + (cg >> 1) : chunk0;
  const uint32_t l0 = lds_addr(lds);
  const uint32_t val = l0, dyl = l0 + 2u * (uint32_t)a.run, lut = dyl + 2 * C::kDyBytes;
  if (threadIdx.x < 16) {
    const u32x2 s = selectors(threadIdx.x);
    *(__attribute__((address_space(3))) u32x2*)(uintptr_t)(lut + 8 * threadIdx.x) = s;
  }
  const int r0 = (int)blockIdx.z * a.per, r1 = min(a.n_stripes, r0 + a.per);
  const uint16_t* const dyb = a.dy + nb0 * (long long)a.rows;

  // The byte offsets of a stripe's values: the workgroup's first chunk, the
  // wave's, and the end.
  struct Run {
    uint32_t t0, tm, t1;
  };
  const const_ptr<uint32_t> co = (const_ptr<uint32_t>)a.chunk_off;
  auto run_of = [&](int r) __attribute__((always_inline)) {
    const size_t at = (size_t)min(r, r1 - 1) * a.chunks;
    return Run{co[at + chunk0], co[at + chunk], co[at + chunk1]};
  };
  // the part q of 3 of stripe r's values
  auto issue_values = [&](int r, int q, const Run& u) __attribute__((always_inline)) {
    if (r >= r1 || u.t1 <= u.t0) return;
    const uint32_t last = u.t1 - u.t0 - 16u;
    const uint32_t to = val + (uint32_t)(r & 1) * (uint32_t)a.run;
    for (uint32_t at = 1024u * (uint32_t)(W * q + wave); at <= last; at += 3u * 1024u * W)
      dma16(a.values, u.t0 + min(at + 16u * (uint32_t)lane, last),
            (uint32_t)__builtin_amdgcn_readfirstlane((int)(to + at)));
  };
  const int piece = (lane & 7) ^ (4 * (wave & 1) + (lane >> 4));
  // the 64 rows of quarter `word` (from the matrix's first) of dY into buffer b: 8
  // tokens a wave and round
  auto issue_dy = [&](int word, int b) __attribute__((always_inline)) {
    if (word >= 4 * r1) return;
    const int m0 = kTM * (word >> 2) + 32 * (word & 3);
#pragma unroll
    for (int i = 0; i < (4 * TB * TG + W - 1) / W; ++i) {
      const int t8 = W * i + wave;
      if (4 * TB * TG % W != 0 && t8 >= 4 * TB * TG) break;
      const uint32_t to = dyl + (uint32_t)(b * C::kDyBytes + t8 * 1024);
      int lane8 = lane >> 3;
      asm volatile("" : "+v"(lane8));  // (keeps the tokens' offsets out of registers between words)
      const uint32_t t = (uint32_t)min(8 * t8 + lane8, last_tok);
      const int m = m0 + 128 * (piece >> 2) + 8 * (piece & 3);
      if constexpr (DYV) {
        if (m0 + 160 <= a.rows || m < a.rows)
          dma16(dyb, (t * (uint32_t)a.rows + (uint32_t)m) * 2u, (uint32_t)__builtin_amdgcn_readfirstlane((int)to));
        else
          *(__attribute__((address_space(3))) u32x4*)(uintptr_t)(to + 16u * (uint32_t)lane) = u32x4{0, 0, 0, 0};
      } else {
        half8 v = half8{0, 0, 0, 0, 0, 0, 0, 0};
        if (m < a.rows) v = load8_inside(dyb + (size_t)t * a.rows + m, a.rows - m);
        *(__attribute__((address_space(3))) half8*)(uintptr_t)(to + 16u * (uint32_t)lane) = v;
      }
    }
  };
  // of a stripe's records: the bits of the lane's 128 rows, and, for a pair of
  // columns, the byte offsets in the chunk of the first value
  struct Rec {
    uint2 w0, w1;
    uint32_t offs;
  };
  const int c16 = lane & 15;
  const unsigned char* const rec_at =
      a.rec + (size_t)chunk * kChunkRecBytes + (4 * (2 * (cg & 1) + (lane >> 4 & 1)) + 2 * half) * kRecBytes;
  auto load_rec1 = [&](int r, Rec& m) __attribute__((always_inline)) {
    const unsigned char* p = rec_at + (size_t)min(r, r1 - 1) * a.chunks * kChunkRecBytes;
    m.w0 = *reinterpret_cast<const uint2*>(p + 8 * c16);
    m.w1 = *reinterpret_cast<const uint2*>(p + kRecBytes + 8 * c16);
    m.offs = *reinterpret_cast<const uint32_t*>(p + 128 + 4 * (c16 >> 1));
  };
  // and from them the bits and the LDS address of the first value
  struct Walk {
    uint32_t mask[4], p;
  };
  auto walk = [&](const Rec& m, int r, const Run& u) __attribute__((always_inline)) {
    return Walk{{m.w0.x, m.w0.y, m.w1.x, m.w1.y},
                val + (uint32_t)(r & 1) * (uint32_t)a.run + (u.tm - u.t0) + ((lane & 1) ? m.offs >> 16 : m.offs & 0xFFFFu)};
  };

  float16v acc[TB];
#pragma unroll
  for (int j = 0; j < TB; ++j) acc[j] = float16v{};
  Run here = run_of(r0), next = run_of(r0 + 1);
  Rec rec;
#pragma unroll
  for (int q = 0; q < 3; ++q) issue_values(r0, q, here);
  issue_dy(4 * r0, 0);
  issue_dy(4 * r0 + 1, 1);
  load_rec1(r0, rec);
  asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)\n\ts_barrier" ::: "memory");
  Walk k = walk(rec, r0, here);
  // Values may be overwritten from the barrier on that follows the stripe's last
  // read of them: its last one, or (32 tokens, whose barriers stand first in a
  // quarter) the next stripe's first.
  constexpr bool kEarly = TB == 1;
  if (!kEarly) issue_values(r0 + 1, 0, next);

  // the tokens' operands are read kLead MFMAs ahead, the values kAhead steps
  // (more for 64 tokens takes the registers of the second workgroup of a CU)
  constexpr int kLead = TB == 2 ? 2 : 4;
  constexpr int kSteps = TB == 1 ? 8 : 2;  // that x holds
  constexpr int kAhead = TB == 1 ? 3 : 2;
  half8 x[kSteps][TB];
  Quad q[kAhead - 1][2];
  Window win;
  u32x2 first;  // the window's first word at the start of a stripe
  const uint32_t db = dyl + (uint32_t)(4096 * TB * tg) + 128u * (uint32_t)(lane & 31);
  auto read_x = [&](int v, int j, int t) __attribute__((always_inline)) {
    const uint32_t place = 16u * (uint32_t)((4 * half + j) ^ (lane >> 1 & 7));
    return *(const __attribute__((address_space(3))) half8*)(uintptr_t)(db + (uint32_t)((v & 1) * C::kDyBytes) + 4096u * t + place);
  };
  // step s of 16 of a stripe
  auto read_q = [&](Walk& w, int s) __attribute__((always_inline)) {
    if (s == 0) first = *(const __attribute__((address_space(3))) u32x2*)(uintptr_t)(w.p & ~7u);
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      const uint32_t b = w.mask[s >> 2] >> (8 * (s & 3) + 4 * i) & 15u;
      q[s % (kAhead - 1)][i].read(w.p, lut + 8u * b);
      w.p += 2u * (uint32_t)__builtin_popcount(b);
    }
  };
  u32x2 w[2];
  auto build = [&](int s, int i) __attribute__((always_inline)) {
    if (s == 0 && i == 0) {
      win.a = first;
      win.at = q[0][0].p & ~7u;
    }
    w[i] = q[s % (kAhead - 1)][i].rows(win);
  };
  read_q(k, 0);
  build(0, 0);
  build(0, 1);
#pragma unroll
  for (int s = 1; s < kAhead; ++s) read_q(k, s);
#pragma unroll
  for (int e = 0; e < kLead; ++e) x[e / TB % kSteps][e % TB] = read_x(0, e / TB, e % TB);

  for (int r = r0; r < r1; ++r) {
    Run after;
    Walk kn;
#pragma unroll
    for (int s = 0; s < 16; ++s) {
      if (s == 8) after = run_of(r + 2);
      const half8 now = __builtin_bit_cast(half8, u32x4{w[0][0], w[0][1], w[1][0], w[1][1]});
      __builtin_amdgcn_sched_barrier(0);
#pragma unroll
      for (int t = 0; t < TB; ++t) {
        const int ahead = s * TB + t + kLead;
        if (ahead % (4 * TB) == 0) {
          // the operands of quarter v have all been read
          const int v = ahead / (4 * TB) - 1;
          asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)\n\ts_barrier" ::: "memory");
          if (v == 2) {
            // the record is there: taken now, for the compiler's own wait for it
            // would count the loads requested below
            asm volatile("" : "+v"(rec.w0.x), "+v"(rec.w0.y), "+v"(rec.w1.x), "+v"(rec.w1.y), "+v"(rec.offs));
            kn = walk(rec, r + 1, next);
          }
          if (v == 1) load_rec1(r + 1, rec);
          issue_dy(4 * r + v + 2, v & 1);
          if (kEarly) {
            if (v < 3) issue_values(r + 1, v, next);
          } else if (v == 3) {
            issue_values(r + 2, 0, after);
          } else if (v < 2) {
            issue_values(r + 1, v + 1, next);
          }
        }
        x[ahead / TB % kSteps][ahead % TB] = read_x(ahead / TB >> 2, ahead / TB & 3, ahead % TB);
        acc[t] = __builtin_amdgcn_mfma_f32_32x32x16_f16(x[s % kSteps][t], now, acc[t], 0, 0, 0);
        if (t == 0) build((s + 1) & 15, 0);
        if (t == (TB > 1 ? 1 : 0)) build((s + 1) & 15, 1);
        if (t == (TB > 2 ? 2 : TB - 1)) read_q(s + kAhead < 16 ? k : kn, (s + kAhead) & 15);
        __builtin_amdgcn_sched_barrier(0);
      }
    }
    k = kn;
    here = next;
    next = after;
  }
  if (!on) return;
  const int col = chunk * kChunkCols + 32 * (cg & 1) + (lane & 31);
#pragma unroll
  for (int t = 0; t < TB; ++t) store_sums(a, acc[t], nb0 + 32 * (TB * tg + t), col);
}

// dX = fp16(sum over the ranges of part[z]), added in order, so that the result
// does not depend on timing; V outputs a lane (4 where the count divides). The sums
// are written and read past the caches (4096 x 4096 at 50 %, 256 tokens, 30.3 -> 29
// us in a graph, 32 tokens 15.3 -> 14.1; larger ones alike).
template <int V>
__global__ __launch_bounds__(kThreads) void grad_reduce_kernel(const float* __restrict__ part, int splits, long long count,
                                                               uint16_t* __restrict__ dx) {
  typedef float floats __attribute__((ext_vector_type(V)));
  const long long stride = (long long)gridDim.x * kThreads;
  for (long long i = (long long)blockIdx.x * kThreads + threadIdx.x; i < count / V; i += stride) {
    floats sum = __builtin_nontemporal_load(reinterpret_cast<const floats*>(part) + i);
#pragma unroll 4
    for (int z = 1; z < splits; ++z) sum += __builtin_nontemporal_load(reinterpret_cast<const floats*>(part + (size_t)z * (size_t)count) + i);
    uint16_t h[V];
#pragma unroll
    for (int e = 0; e < V; ++e) {
      const float v = sum[e];
      h[e] = __half_as_ushort(__float2half_rn(v));
    }
    __builtin_memcpy(dx + V * i, h, 2 * V);
  }
}

// ---------------------------------------------------------------------------
// Host side.

using namespace spdp;

constexpr int kLdsMax = 160 * 1024;

// The forms: blocks of 32 tokens of a wave, groups of 32 columns and groups of
// tokens of a workgroup; and what a quarter of a stripe (64 rows) takes, us, with
// one, two, ... workgroups on a CU (0: LDS or registers hold no more).
struct Form {
  int tb, cg, tg;
  float us[4];
  int tokens() const { return 32 * tb * tg; }
  int lds(const spdp_matrix* h) const { return 2 * h->run_bytes[cg / 8] + 2 * tokens() * 128 + 256; }
};
constexpr Form kForms[] = {
    {1, 4, 1, {0.62f, 0.83f, 1.18f, 1.34f}}, {2, 4, 1, {0.75f, 0.90f, 1.14f, 0.0f}},
    {4, 4, 1, {0.98f, 1.74f, 0.0f, 0.0f}},   {4, 4, 2, {1.27f, 0.0f, 0.0f, 0.0f}},
    {1, 8, 1, {0.76f, 1.09f, 0.0f, 0.0f}},   {2, 8, 1, {0.90f, 1.22f, 0.0f, 0.0f}},
    {4, 8, 1, {1.13f, 0.0f, 0.0f, 0.0f}},    {8, 8, 1, {1.75f, 0.0f, 0.0f, 0.0f}}};
constexpr int kNumForms = sizeof(kForms) / sizeof(kForms[0]);

struct GradPlan {
  int form;  // -1: plain
  long long tiles;
  int blocks, per, splits;
};

int env_int(const char* name, int otherwise) {
  const char* env = std::getenv(name);
  return env ? std::atoi(env) : otherwise;
}

// us of a form with `splits` ranges of the stripes, by the model that the table
// above is fitted to (1144 launches of 7 matrices at 16 to 2048 tokens, 8 % rms; the
// choice loses 2.4 % on average to the best of all forms and splits): rounds of
// workgroups, 1 us each; 1.9 us and 8 bytes per sum at 5.7 TB/s for the second
// launch that adds the ranges.
float model_us(const spdp_matrix* h, const Form& f, long long wgs, int per, int splits, long long n_tokens, int cus) {
  int most = 1;
  while (most < 4 && f.us[most] > 0.0f && (most + 1) * f.lds(h) <= kLdsMax) ++most;
  const long long full = wgs / ((long long)cus * most), rest = wgs - full * cus * most;
  const int k = (int)((rest + cus - 1) / cus);  // workgroups on a CU in the last round
  float us = (float)full * (4.0f * (float)per * f.us[most - 1] + 0.7f);
  if (k > 0) us += 4.0f * (float)per * f.us[k - 1] + 1.0f;
  if (splits > 1) us += 1.9f + (float)splits * (float)n_tokens * (float)h->cols * 8.0f / 5.7e6f;
  return us;
}

// The form and split of the least modelled time, within 256 MB of partial sums.
// SPDP_GRAD_FORM (a testing aid) forces a form by its place in the table, or the
// plain one (-1, and where the forced one's LDS does not fit), SPDP_GRAD_SPLITS the
// ranges.
void plan_grad(const spdp_matrix* h, long long n_tokens, GradPlan* p) {
  const int cus = std::max(1, h->cus);
  const int forced_splits = env_int("SPDP_GRAD_SPLITS", 0), forced_form = env_int("SPDP_GRAD_FORM", -2);
  const long long stripes = h->n_stripes;
  p->form = -1;
  p->tiles = (n_tokens + 127) / 128;
  p->blocks = (int)((h->cols + 63) / 64);
  float least = 0.0f;
  for (int i = 0; i < kNumForms; ++i) {
    const Form& f = kForms[i];
    if ((forced_form > -2 && forced_form != i) || h->d_rec == nullptr || f.lds(h) > kLdsMax ||
        std::min<long long>(n_tokens, f.tokens()) * h->rows * 2 > 1ll << 32 || (n_tokens + f.tokens() - 1) / f.tokens() > 65535)
      continue;
    const long long tiles = (n_tokens + f.tokens() - 1) / f.tokens();
    const int blocks = (int)((h->cols + 32 * f.cg - 1) / (32 * f.cg));
    for (int want = forced_splits > 0 ? (int)std::min<long long>(forced_splits, stripes) : 1;; ++want) {
      const int per = (int)((stripes + want - 1) / want), splits = (int)((stripes + per - 1) / per);
      const float us = model_us(h, f, tiles * blocks * splits, per, splits, n_tokens, cus);
      if (p->form < 0 || us < least) {
        least = us;
        *p = GradPlan{i, tiles, blocks, per, splits};
      }
      if (forced_splits > 0 || want >= 16 || want >= stripes || (float)(want + 1) * n_tokens * h->cols * 4.0f > 256e6f) break;
    }
  }
  if (p->form >= 0) return;
  const long long wgs = p->tiles * p->blocks;
  const long long want =
      std::min<long long>(stripes, forced_splits > 0 ? forced_splits : std::max<long long>(1, std::min<long long>(16, cus / wgs)));
  p->per = (int)((stripes + want - 1) / want);
  p->splits = (int)((stripes + p->per - 1) / p->per);
}

size_t part_bytes(const spdp_matrix* h, long long n_tokens, const GradPlan& p) {
  return p.splits > 1 ? (size_t)p.splits * n_tokens * h->cols * 4 : 0;
}

template <int TB, int CG, int TG, bool DYV>
hipError_t launch_form(const GradArgs& a, dim3 grid, hipStream_t st) {
  const int lds = GradCfg<TB, CG, TG>::lds(a.run);
  const auto kernel = grad_kernel<TB, CG, TG, DYV>;
  if (lds > 64 * 1024) {
    const hipError_t e =
        hipFuncSetAttribute(reinterpret_cast<const void*>(kernel), hipFuncAttributeMaxDynamicSharedMemorySize, lds);
    if (e != hipSuccess) return e;
  }
  hipLaunchKernelGGL(kernel, grid, dim3(64 * CG * TG), lds, st, a);
  return hipGetLastError();
}
template <int I>
hipError_t launch_forms(int form, const GradArgs& a, dim3 grid, hipStream_t st) {
  if constexpr (I < kNumForms) {
    constexpr Form f = kForms[I];
    if (form != I) return launch_forms<I + 1>(form, a, grid, st);
    return a.rows % 8 == 0 ? launch_form<f.tb, f.cg, f.tg, true>(a, grid, st) : launch_form<f.tb, f.cg, f.tg, false>(a, grid, st);
  }
  return hipErrorInvalidValue;
}

int check(const spdp_matrix* h, int64_t n_tokens) {
  if (!h) return fail(SPDP_ERR_INVALID_ARG, "handle is NULL");
  if (h->device < 0) return fail(SPDP_ERR_INVALID_ARG, "handle has no device copy");
  if (n_tokens < 1) return fail(SPDP_ERR_INVALID_ARG, "n_tokens must be at least 1");
  if (h->value_bits < 16) return fail(SPDP_ERR_UNSUPPORTED, "the gradient takes fp16 Values, not codes");
  if (h->tile_m != kTM || h->tile_k < 16)
    return fail(SPDP_ERR_UNSUPPORTED, "the gradient needs tile_m = 256 and tile_k >= 16");
  if (n_tokens > 65535ll * 32) return fail(SPDP_ERR_UNSUPPORTED, "more than 65535 x 32 tokens");
  return SPDP_OK;
}

int spmm_grad(spdp_handle_t h, const uint16_t* dY, int64_t n_tokens, uint16_t* dX, void* workspace, size_t workspace_bytes,
              void* stream) {
  int st = check(h, n_tokens);
  if (st != SPDP_OK) return st;
  if (!dY || !dX) return fail(SPDP_ERR_INVALID_ARG, "dY or dX is NULL");
  if ((reinterpret_cast<uintptr_t>(dY) | reinterpret_cast<uintptr_t>(dX)) & 15)
    return fail(SPDP_ERR_INVALID_ARG, "dY and dX must be 16-byte aligned");
  if (overlap(dY, (size_t)n_tokens * h->rows * 2, dX, (size_t)n_tokens * h->cols * 2))
    return fail(SPDP_ERR_INVALID_ARG, "dY and dX overlap");
  int dev = -1;
  hipError_t e = hipGetDevice(&dev);
  if (e != hipSuccess) return hip_fail(e, "hipGetDevice");
  if (dev != h->device) return fail(SPDP_ERR_INVALID_ARG, "current device differs from the handle's");
  GradPlan p;
  plan_grad(h, n_tokens, &p);
  st = check_workspace(workspace, workspace_bytes, part_bytes(h, n_tokens, p));
  if (st != SPDP_OK) return st;
  GradArgs a;
  std::memset(&a, 0, sizeof(a));
  a.tile_offset = static_cast<const uint32_t*>(h->d_tile_offset);
  a.col_info = static_cast<const uint32_t*>(h->d_col_info);
  a.bitmap = static_cast<const uint64_t*>(h->d_bitmap);
  a.rec = static_cast<const unsigned char*>(h->d_rec);
  a.chunk_off = static_cast<const uint32_t*>(h->d_chunk_off);
  a.values = static_cast<const uint16_t*>(h->d_values);
  a.dy = dY;
  a.dx = dX;
  a.part = static_cast<float*>(workspace);
  a.n_tokens = n_tokens;
  a.rows = (int)h->rows;
  a.cols = (int)h->cols;
  a.tk_log2 = __builtin_ctz((unsigned)h->tile_k);
  a.n_colblocks = (int)h->n_colblocks;
  a.n_stripes = (int)h->n_stripes;
  a.per = p.per;
  a.chunks = h->chunks;
  a.run = p.form >= 0 ? h->run_bytes[kForms[p.form].cg / 8] : 0;
  auto s = static_cast<hipStream_t>(stream);
  const dim3 grid((unsigned)p.blocks, (unsigned)p.tiles, (unsigned)p.splits);
  if (p.form >= 0) {
    e = launch_forms<0>(p.form, a, grid, s);
  } else {
    hipLaunchKernelGGL(grad_plain_kernel, grid, dim3(kThreads), 0, s, a);
    e = hipGetLastError();
  }
  if (e == hipSuccess && p.splits > 1) {
    const long long count = n_tokens * h->cols;
    const bool four = count % 4 == 0;
    const unsigned wgs = (unsigned)std::min<long long>(8192, ((four ? count / 4 : count) + kThreads - 1) / kThreads);
    if (four)
      hipLaunchKernelGGL(grad_reduce_kernel<4>, dim3(wgs), dim3(kThreads), 0, s, a.part, p.splits, count, dX);
    else
      hipLaunchKernelGGL(grad_reduce_kernel<1>, dim3(wgs), dim3(kThreads), 0, s, a.part, p.splits, count, dX);
    e = hipGetLastError();
  }
  return e == hipSuccess ? SPDP_OK : hip_fail(e, "kernel launch");
}

}  // namespace

extern "C" {

int spdp_spmm_grad_workspace(spdp_handle_t h, int64_t n_tokens, size_t* bytes) {
  return guarded([&] {
    if (!bytes) return fail(SPDP_ERR_INVALID_ARG, "bytes is NULL");
    const int st = check(h, n_tokens);
    if (st != SPDP_OK) return st;
    GradPlan p;
    plan_grad(h, n_tokens, &p);
    *bytes = part_bytes(h, n_tokens, p);
    return (int)SPDP_OK;
  });
}

int spdp_spmm_grad(spdp_handle_t h, const uint16_t* dY, int64_t n_tokens, uint16_t* dX, void* workspace,
                   size_t workspace_bytes, void* stream) {
  return guarded([&] { return spmm_grad(h, dY, n_tokens, dX, workspace, workspace_bytes, stream); });
}

}  // extern "C"
