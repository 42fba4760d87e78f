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

#include <hip/hip_fp16.h>
#include <hip/hip_runtime.h>

#include <algorithm>
#include <cstdlib>
#include <cstring>

#include "internal.h"
#include "lanes.h"
#include "launch.h"

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
  int chunks, slot;
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
      part[n * (long long)a.cols + col] = acc[e];
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
// The form for handles with word records. Four waves own 128 columns (two
// chunks) and 32 TB tokens; wave w has the columns 32 w .. + 31, lane l column
// l mod 32 and, of each 64-row word, the rows 32 (l / 32) .. + 31. Per four
// rows a lane reads the next four values of its column from LDS (at any 2-byte
// address: as many are used as the four bits of the bitmap word have ones) and
// puts them into their places with two byte permutations, whose selectors a
// table of 16 entries holds. Eight rows are an operand of
// v_mfma_f32_32x32x16_f16; the tokens' operands come from LDS in the same order
// of rows.
//
// Per stripe the two chunks' values (one contiguous run) arrive by DMA one
// stripe ahead, a quarter with each word; per word the tokens' 64 rows of dY,
// one word ahead, 16-byte piece p of token t at place p ^ (t mod 8).

template <int TB>
struct GradCfg {
  static constexpr int kTokens = 32 * TB;
  static constexpr int kDyBytes = kTokens * 128;
  static int lds(int slot) { return 4 * slot + 2 * kDyBytes + 256; }
};

typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));

__device__ __forceinline__ u32x2 lds_read8(uint32_t at) {
  u32x2 v;
  __builtin_memcpy(&v, (const __attribute__((address_space(3))) unsigned char*)(uintptr_t)at, 8);
  return v;
}

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
template <int TB, bool DYV>
__global__ __launch_bounds__(kThreads) void grad_kernel(GradArgs a) {
  using C = GradCfg<TB>;
  extern __shared__ __attribute__((aligned(1024))) unsigned char lds[];
  const int lane = threadIdx.x & 63;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int half = lane >> 5;
  const long long nb0 = (long long)blockIdx.y * C::kTokens;
  const int last_tok = (int)min(a.n_tokens - nb0, (long long)C::kTokens) - 1;
  const int chunk0 = 2 * (int)blockIdx.x;
  const int chunk1 = min(chunk0 + 2, a.chunks);
  const int chunk = chunk0 + (wave >> 1);
  const bool on = chunk < chunk1;  // the last workgroup's second chunk may be none
  const uint32_t l0 = lds_addr(lds);
  const uint32_t val = l0, dyl = l0 + 4u * (uint32_t)a.slot, lut = dyl + 2 * C::kDyBytes;
  if (threadIdx.x < 16) {
    const u32x2 s = selectors(threadIdx.x);
    *(__attribute__((address_space(3))) u32x2*)(uintptr_t)(lut + 8 * threadIdx.x) = s;
  }
  const int r0 = (int)blockIdx.z * a.per, r1 = min(a.n_stripes, r0 + a.per);
  const uint16_t* const dyb = a.dy + nb0 * (long long)a.rows;

  // the part `q` of 4 of stripe r's values, [t0, t1) of the values' bytes
  auto issue_values = [&](int r, int q, uint32_t t0, uint32_t t1) __attribute__((always_inline)) {
    if (t1 <= t0) return;
    const uint32_t last = t1 - t0 - 16u;
    const uint32_t to = val + (uint32_t)(r & 1) * 2u * (uint32_t)a.slot;
    for (uint32_t at = 1024u * (uint32_t)(4 * q + wave); at <= last; at += 16384u)
      dma16(a.values, t0 + min(at + 16u * (uint32_t)lane, last),
            (uint32_t)__builtin_amdgcn_readfirstlane((int)(to + at)));
  };
  const int piece = (lane & 7) ^ (lane >> 3);
  // 64 rows of dY from row m0 on into buffer b
  auto issue_dy = [&](int m0, int b) __attribute__((always_inline)) {
#pragma unroll
    for (int i = 0; i < TB; ++i) {
      const uint32_t to = dyl + (uint32_t)(b * C::kDyBytes + (32 * i + 8 * wave) * 128);
      const uint32_t t = (uint32_t)min(32 * i + 8 * wave + (lane >> 3), last_tok);
      const int m = m0 + 8 * piece;
      if constexpr (DYV) {
        if (m < a.rows)
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
  // the lane's record of stripe r, word v: its column's word and the byte
  // offset of the word's first value in the chunk
  struct Rec {
    uint64_t word;
    uint32_t off;
  };
  const int c16 = lane & 15;
  const int group = 2 * (wave & 1) + (lane >> 4 & 1);
  auto load_rec1 = [&](int r, int v, Rec& m) __attribute__((always_inline)) {
    const unsigned char* p =
        a.rec + ((size_t)r * a.chunks + (on ? chunk : chunk0)) * kChunkRecBytes + (4 * group + v) * kRecBytes;
    m.word = *reinterpret_cast<const uint64_t*>(p + 8 * c16);
    m.off = *reinterpret_cast<const uint16_t*>(p + 128 + 2 * c16);
  };

  float16v acc[TB];
#pragma unroll
  for (int j = 0; j < TB; ++j) acc[j] = float16v{};
  const const_ptr<uint32_t> co = (const_ptr<uint32_t>)a.chunk_off;

  Rec cur, nxt;
  uint32_t t0 = co[(size_t)r0 * a.chunks + chunk0], tm = co[(size_t)r0 * a.chunks + (on ? chunk : chunk0)],
           t1 = co[(size_t)r0 * a.chunks + chunk1];
#pragma unroll
  for (int q = 0; q < 4; ++q) issue_values(r0, q, t0, t1);
  issue_dy(r0 * kTM, 0);
  load_rec1(r0, 0, cur);
  for (int r = r0; r < r1; ++r) {
    // the chunk's values in LDS
    const uint32_t mine = val + (uint32_t)(r & 1) * 2u * (uint32_t)a.slot + (tm - t0);
    const bool more = r + 1 < r1;
    uint32_t n0 = 0, nm = 0, n1 = 0;
    if (more) {
      const size_t at = (size_t)(r + 1) * a.chunks;
      n0 = co[at + chunk0];
      nm = co[at + (on ? chunk : chunk0)];
      n1 = co[at + chunk1];
    }
#pragma unroll
    for (int v = 0; v < 4; ++v) {
      asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)\n\ts_barrier" ::: "memory");
      if (v < 3)
        issue_dy(r * kTM + 64 * (v + 1), (v + 1) & 1);
      else if (more)
        issue_dy((r + 1) * kTM, 0);
      if (more) issue_values(r + 1, v, n0, n1);
      if (v < 3)
        load_rec1(r, v + 1, nxt);
      else if (more)
        load_rec1(r + 1, 0, nxt);
      if (on) {
        const uint32_t lo = (uint32_t)cur.word;
        const uint32_t mask = half ? (uint32_t)(cur.word >> 32) : lo;
        uint32_t p = mine + cur.off + (half ? 2u * (uint32_t)__builtin_popcount(lo) : 0u);
        const uint32_t db = dyl + (uint32_t)((v & 1) * C::kDyBytes) + 128u * (uint32_t)(lane & 31);
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          const uint32_t b0 = mask >> (8 * j) & 15u, b1 = mask >> (8 * j + 4) & 15u;
          const uint32_t p1 = p + 2u * (uint32_t)__builtin_popcount(b0);
          const u32x2 v0 = lds_read8(p), v1 = lds_read8(p1);
          p = p1 + 2u * (uint32_t)__builtin_popcount(b1);
          const u32x2 s0 = *(const __attribute__((address_space(3))) u32x2*)(uintptr_t)(lut + 8u * b0);
          const u32x2 s1 = *(const __attribute__((address_space(3))) u32x2*)(uintptr_t)(lut + 8u * b1);
          const half8 w = __builtin_bit_cast(
              half8, u32x4{__builtin_amdgcn_perm(v0[1], v0[0], s0[0]), __builtin_amdgcn_perm(v0[1], v0[0], s0[1]),
                           __builtin_amdgcn_perm(v1[1], v1[0], s1[0]), __builtin_amdgcn_perm(v1[1], v1[0], s1[1])});
          const uint32_t place = 16u * (uint32_t)((4 * half + j) ^ (lane & 7));
#pragma unroll
          for (int t = 0; t < TB; ++t) {
            const half8 x = *(const __attribute__((address_space(3))) half8*)(uintptr_t)(db + 4096u * t + place);
            acc[t] = __builtin_amdgcn_mfma_f32_32x32x16_f16(x, w, acc[t], 0, 0, 0);
          }
        }
      }
      cur = nxt;
    }
    t0 = n0;
    tm = nm;
    t1 = n1;
  }
  if (!on) return;
  const int col = chunk * kChunkCols + 32 * (wave & 1) + (lane & 31);
#pragma unroll
  for (int t = 0; t < TB; ++t) store_sums(a, acc[t], nb0 + 32 * t, col);
}

// ---------------------------------------------------------------------------
// Host side.

using spdp::fail;

int hip_fail(hipError_t e, const char* what) {
  return fail(SPDP_ERR_HIP, std::string(what) + ": " + hipGetErrorString(e));
}

constexpr int kLdsMax = 160 * 1024;

struct GradPlan {
  int tb;  // 0: plain
  long long tiles;
  int blocks, per, splits;
};

int lds_bytes(int tb, int slot) {
  return tb == 1 ? GradCfg<1>::lds(slot) : tb == 2 ? GradCfg<2>::lds(slot) : tb == 4 ? GradCfg<4>::lds(slot) : GradCfg<8>::lds(slot);
}

void plan_grad(const spdp_matrix* h, long long n_tokens, GradPlan* p) {
  const int cus = std::max(1, h->cus);
  int forced = 0, forced_tb = -1;
  if (const char* env = std::getenv("SPDP_GRAD_SPLITS")) forced = std::max(1, std::atoi(env));
  if (const char* env = std::getenv("SPDP_GRAD_TOKENS")) forced_tb = std::atoi(env) / 32;
  const long long stripes = h->n_stripes;
  auto fits = [&](int tb) {
    return h->d_rec != nullptr && lds_bytes(tb, h->chunk_bytes) <= kLdsMax &&
           std::min<long long>(n_tokens, 32 * tb) * h->rows * 2 <= 1ll << 32 && (n_tokens + 32 * tb - 1) / (32 * tb) <= 65535;
  };
  auto fill = [&](int tb) {
    p->tb = tb;
    const int tokens = tb ? 32 * tb : 128;
    p->tiles = (n_tokens + tokens - 1) / tokens;
    p->blocks = tb ? (h->chunks + 1) / 2 : (int)((h->cols + 63) / 64);
    const long long wgs = p->tiles * p->blocks;
    const long long want = forced ? forced : std::max<long long>(1, std::min<long long>(16, cus / wgs));
    p->per = (int)((stripes + std::min(want, stripes) - 1) / std::min(want, stripes));
    p->splits = (int)((stripes + p->per - 1) / p->per);
  };
  if (forced_tb >= 0) {
    const int tb = forced_tb >= 8 ? 8 : forced_tb >= 4 ? 4 : forced_tb >= 2 ? 2 : forced_tb;
    fill(tb > 0 && fits(tb) ? tb : 0);
    return;
  }
  int best = 0;
  for (int tb = 1; tb <= 8; tb *= 2) {
    if (!fits(tb)) continue;
    if (best == 0 || 32 * tb <= n_tokens) best = tb;
  }
  fill(best);
}

size_t part_bytes(const spdp_matrix* h, long long n_tokens, const GradPlan& p) {
  return p.splits > 1 ? (size_t)p.splits * n_tokens * h->cols * 4 : 0;
}

template <int TB, bool DYV>
hipError_t launch_form(const GradArgs& a, dim3 grid, hipStream_t st) {
  const int lds = GradCfg<TB>::lds(a.slot);
  const auto kernel = grad_kernel<TB, DYV>;
  if (lds > 64 * 1024) {
    const hipError_t e =
        hipFuncSetAttribute(reinterpret_cast<const void*>(kernel), hipFuncAttributeMaxDynamicSharedMemorySize, lds);
    if (e != hipSuccess) return e;
  }
  hipLaunchKernelGGL(kernel, grid, dim3(kThreads), lds, st, a);
  return hipGetLastError();
}
template <int TB>
hipError_t launch_tb(const GradArgs& a, dim3 grid, hipStream_t st) {
  return a.rows % 8 == 0 ? launch_form<TB, true>(a, grid, st) : launch_form<TB, false>(a, grid, st);
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
  const int st = check(h, n_tokens);
  if (st != SPDP_OK) return st;
  if (!dY || !dX) return fail(SPDP_ERR_INVALID_ARG, "dY or dX is NULL");
  if ((reinterpret_cast<uintptr_t>(dY) | reinterpret_cast<uintptr_t>(dX)) & 15)
    return fail(SPDP_ERR_INVALID_ARG, "dY and dX must be 16-byte aligned");
  const uintptr_t y0 = reinterpret_cast<uintptr_t>(dY), y1 = y0 + (uintptr_t)n_tokens * h->rows * 2;
  const uintptr_t x0 = reinterpret_cast<uintptr_t>(dX), x1 = x0 + (uintptr_t)n_tokens * h->cols * 2;
  if (x0 < y1 && y0 < x1) return fail(SPDP_ERR_INVALID_ARG, "dY and dX overlap");
  int dev = -1;
  hipError_t e = hipGetDevice(&dev);
  if (e != hipSuccess) return hip_fail(e, "hipGetDevice");
  if (dev != h->device) return fail(SPDP_ERR_INVALID_ARG, "current device differs from the handle's");
  GradPlan p;
  plan_grad(h, n_tokens, &p);
  const size_t need = part_bytes(h, n_tokens, p);
  if (need > 0) {
    if (!workspace) return fail(SPDP_ERR_INVALID_ARG, "workspace is NULL");
    if (reinterpret_cast<uintptr_t>(workspace) & 255) return fail(SPDP_ERR_INVALID_ARG, "workspace must be 256-byte aligned");
    if (workspace_bytes < need)
      return fail(SPDP_ERR_INVALID_ARG,
                  "workspace of " + std::to_string(workspace_bytes) + " bytes, " + std::to_string(need) + " needed");
  }
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
  a.slot = h->chunk_bytes;
  auto s = static_cast<hipStream_t>(stream);
  const dim3 grid((unsigned)p.blocks, (unsigned)p.tiles, (unsigned)p.splits);
  switch (p.tb) {
    case 1: e = launch_tb<1>(a, grid, s); break;
    case 2: e = launch_tb<2>(a, grid, s); break;
    case 4: e = launch_tb<4>(a, grid, s); break;
    case 8: e = launch_tb<8>(a, grid, s); break;
    default:
      hipLaunchKernelGGL(grad_plain_kernel, grid, dim3(kThreads), 0, s, a);
      e = hipGetLastError();
  }
  if (e == hipSuccess && p.splits > 1)
    e = spdp::launch_reduce(a.part, p.splits, n_tokens * h->cols, dX, s);
  return e == hipSuccess ? SPDP_OK : hip_fail(e, "kernel launch");
}

template <class F>
int guarded(F f) {
  try {
    spdp::clear_error();
    return f();
  } catch (...) {  // a message found no memory
    return SPDP_ERR_OOM;
  }
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
