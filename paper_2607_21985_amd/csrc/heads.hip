// Norm and position rotation of the heads of queries and keys, one pass.
//
// A head v of `dim` numbers becomes n = v rsqrt(mean v^2 + eps) w (where there
// are weights w), and each pair (p, q) of its leading 2 half numbers becomes
// (p c - q s, p s + q c) with the angles of the token's position. Backward: g =
// the rotation by the negative angle of dy; dw = sum over heads and tokens of
// g v r with r = rsqrt(...); dv = r (w g - v r^2 mean(w g v)).
//
// Bound by memory: each number is read and written once. A group of lanes
// owns a head and each lane the two vectors of V numbers that rotate into one
// another (half-split pairs) or any two (neighbours as pairs, and the rest of
// the head), so the rotation needs no exchange between lanes. A wave keeps its
// token's angles in registers for several heads. Measured: 4096 tokens of 32 + 32
// heads of 128, 23 us, 5.8 TB/s (a copy has 5.2); backward, 2048 tokens of
// 40 + 8 heads of 96, 18 us, 3.1 TB/s, with three workgroups of long chains a CU.

#include <hip/hip_fp16.h>
#include <hip/hip_runtime.h>

#include <algorithm>
#include <cstring>

#include "calls.h"

namespace {

constexpr int kMaxInputs = 8;
constexpr int kThreads = 256;
constexpr int kWaves = 4;
constexpr int kMaxDim = 512;

struct HeadsInput {
  const uint16_t* x;
  const uint16_t* w;   // NULL: no norm
  const uint16_t* dy;  // backward
  uint16_t* y;         // or dx
  float* part;         // backward with weights: [workgroup of this input][dim]
  int heads;
  int wg0;             // the input's first workgroup
  int per;             // heads of a group of lanes, one after another
};
struct HeadsArgs {
  HeadsInput m[kMaxInputs];
  const int* pos;
  const float* cosine;
  const float* sine;
  float eps;
  int inputs;
  int n_tokens;
  int positions;
  int dim, half;
  int lanes;  // of a head: a power of two
};

// 16 bytes at any address of fp16
typedef uint32_t Vec __attribute__((ext_vector_type(4), aligned(2)));

// V fp16 as they are in memory (words of two, so that a pending load takes no more
// registers than its bytes)
template <int V>
struct Raw {
  uint32_t w[(V + 1) / 2];
  template <bool ONCE>
  __device__ __forceinline__ void load(const uint16_t* p) {
    if constexpr (ONCE) {
      const Vec v = __builtin_nontemporal_load(reinterpret_cast<const Vec*>(p));
      __builtin_memcpy(w, &v, 2 * V);
    } else {
      __builtin_memcpy(w, p, 2 * V);
    }
  }
  __device__ __forceinline__ void clear() {
#pragma unroll
    for (int e = 0; e < (V + 1) / 2; ++e) w[e] = 0;
  }
  __device__ __forceinline__ float operator[](int e) const {
    return __half2float(__ushort_as_half((uint16_t)(w[e / 2] >> (e % 2 * 16))));
  }
};
template <int V, bool ONCE>
__device__ __forceinline__ void store_v(uint16_t* p, const float (&v)[V]) {
  uint16_t h[V];
#pragma unroll
  for (int e = 0; e < V; ++e) h[e] = __half_as_ushort(__float2half_rn(v[e]));
  if constexpr (ONCE) {
    Vec v;
    __builtin_memcpy(&v, h, 2 * V);
    __builtin_nontemporal_store(v, reinterpret_cast<Vec*>(p));
  } else {
    __builtin_memcpy(p, h, 2 * V);
  }
}

// A lane's place in a head: the vectors at a and b (past the end: none), and
// whether they rotate. PAIRS: pairs are neighbours, within a and within b; else
// a rotates with b.
struct Slot {
  int a, b;
  bool turns;
};
template <int V, bool PAIRS>
__device__ __forceinline__ Slot slot_of(int s, int half) {
  if (!PAIRS && s < half / V) return Slot{s * V, half + s * V, true};
  const int from = PAIRS ? 0 : half / V;
  const int at = (PAIRS ? 0 : 2 * half) + 2 * V * (s - from);
  return Slot{at, at + V, PAIRS};
}

// The rotation of a slot's vectors by the angle's cosine and (sign times) sine;
// numbers past the leading ones turn by none.
template <int V, bool PAIRS>
struct Turn {
  static constexpr int kAngles = V;  // PAIRS: V / 2 of a, V / 2 of b
  float c[kAngles], s[kAngles];
  __device__ __forceinline__ void load(const HeadsArgs& a, const Slot& t, long long pos, float sign) {
    const float* const tc = a.cosine + pos * a.half;
    const float* const ts = a.sine + pos * a.half;
    const int at = PAIRS ? t.a / 2 : t.a;  // (b's angles follow a's)
#pragma unroll
    for (int e = 0; e < V; ++e) {
      c[e] = 1.0f;
      s[e] = 0.0f;
    }
    if (t.turns && at + V <= a.half) {
      __builtin_memcpy(c, tc + at, 4 * V);
      __builtin_memcpy(s, ts + at, 4 * V);
    } else if (PAIRS && at < a.half) {  // the leading numbers end within the vector
#pragma unroll
      for (int e = 0; e < V; ++e)
        if (at + e < a.half) {
          c[e] = tc[at + e];
          s[e] = ts[at + e];
        }
    }
#pragma unroll
    for (int e = 0; e < V; ++e) s[e] *= sign;
  }
  __device__ __forceinline__ void apply(float (&x)[2][V]) const {
#pragma unroll
    for (int e = 0; e < V; ++e) {
      float& first = PAIRS ? x[2 * e / V][2 * e % V] : x[0][e];
      float& second = PAIRS ? x[2 * e / V][2 * e % V + (V > 1)] : x[1][e];
      const float p = first, q = second;
      first = p * c[e] - q * s[e];
      second = q * c[e] + p * s[e];
    }
  }
};

// The sum over the 2^k lanes of a head, in each of them; all lanes are active. Lanes
// that hold equal sums already may be met in any order, so that the mirrored rows
// of the data-parallel moves will do.
template <int CTRL>
__device__ __forceinline__ float moved(float v) {
  return __int_as_float(__builtin_amdgcn_update_dpp(0, __float_as_int(v), CTRL, 0xf, 0xf, true));
}
__device__ __forceinline__ float head_sum(float v, int lanes) {
  if (lanes > 1) v += moved<0xb1>(v);    // 1 0 3 2
  if (lanes > 2) v += moved<0x4e>(v);    // 2 3 0 1
  if (lanes > 4) v += moved<0x141>(v);   // 8 lanes backwards
  if (lanes > 8) v += moved<0x140>(v);   // 16 lanes backwards
  if (lanes > 16) v += __shfl_xor(v, 16);
  if (lanes > 32) v += __shfl_xor(v, 32);
  return v;
}

// A workgroup of an input: its groups of lanes take `per` heads of a token
// each, the groups of a wave all of one token. ONCE: outputs (backward: inputs,
// too) go past the caches, which cannot hold them.
template <int V, int R, bool PAIRS, bool BACK, bool ONCE>
__global__ __launch_bounds__(kThreads) void heads_kernel(HeadsArgs a) {
  int which = 0;
  while (which + 1 < a.inputs && (int)blockIdx.x >= a.m[which + 1].wg0) ++which;
  const HeadsInput& m = a.m[which];
  const int lane = threadIdx.x & 63;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int groups = 64 / a.lanes;
  const int group = lane / a.lanes, sub = lane % a.lanes;
  const int chunk = groups * m.per;  // heads of a wave's round
  const int chunks = (m.heads + chunk - 1) / chunk;
  const bool norm = m.w != nullptr;
  const float inv_dim = 1.0f / (float)a.dim;

  Slot t[R];
  float w[R][2][V];
  float dw[R][2][V];
#pragma unroll
  for (int r = 0; r < R; ++r) {
    t[r] = slot_of<V, PAIRS>(sub + 64 * r, a.half);
#pragma unroll
    for (int k = 0; k < 2; ++k) {
      const int from = k == 0 ? t[r].a : t[r].b;
      Raw<V> weights;
      weights.clear();
      if (norm && from < a.dim) weights.template load<false>(m.w + from);
#pragma unroll
      for (int e = 0; e < V; ++e) {
        w[r][k][e] = norm ? weights[e] : 1.0f;
        dw[r][k][e] = 0.0f;
      }
    }
  }
  const int wgs = (which + 1 < a.inputs ? a.m[which + 1].wg0 : (int)gridDim.x) - m.wg0;
  const long long rounds = (long long)a.n_tokens * chunks;
  for (long long q = ((long long)blockIdx.x - m.wg0) * kWaves + wave; q < rounds; q += (long long)wgs * kWaves) {
    const int tok = (int)(q / chunks);
    const int h0 = (int)(q % chunks) * chunk;
    const int pos = a.pos[tok];
    if ((unsigned)pos >= (unsigned)a.positions) {  // a padding token
      if constexpr (BACK) {
        // (zeros as such: products with no numbers would not be where a weight is NaN)
        const float zeros[V] = {};
        for (int h = h0 + group; h < min(h0 + chunk, m.heads); h += groups) {
          const size_t at = ((size_t)tok * m.heads + h) * a.dim;
#pragma unroll
          for (int r = 0; r < R; ++r) {
            if (t[r].a < a.dim) store_v<V, ONCE>(m.y + at + t[r].a, zeros);
            if (t[r].b < a.dim) store_v<V, ONCE>(m.y + at + t[r].b, zeros);
          }
        }
      }
      continue;
    }
    Turn<V, PAIRS> u[R];
#pragma unroll
    for (int r = 0; r < R; ++r) u[r].load(a, t[r], pos, BACK ? -1.0f : 1.0f);
    // a head's numbers, requested a head ahead
    Raw<V> nx[R][2], ng[R][2];
    auto request = [&](int h) __attribute__((always_inline)) {
      const size_t at = ((size_t)tok * m.heads + h) * a.dim;
#pragma unroll
      for (int r = 0; r < R; ++r)
#pragma unroll
        for (int k = 0; k < 2; ++k) {
          const int from = k == 0 ? t[r].a : t[r].b;
          nx[r][k].clear();
          if (BACK) ng[r][k].clear();
          if (h < m.heads && from < a.dim) {
            if (!BACK || norm) nx[r][k].template load<ONCE && BACK>(m.x + at + from);
            if (BACK) ng[r][k].template load<ONCE>(m.dy + at + from);
          }
        }
    };
    request(h0 + group);
    for (int i = 0; i < m.per; ++i) {
      const int h = h0 + i * groups + group;
      const bool on = h < m.heads;
      const size_t at = ((size_t)tok * m.heads + (on ? h : 0)) * a.dim;
      float x[R][2][V], g[R][2][V];
      float sum = 0.0f, dot = 0.0f;
#pragma unroll
      for (int r = 0; r < R; ++r)
#pragma unroll
        for (int k = 0; k < 2; ++k)
#pragma unroll
          for (int e = 0; e < V; ++e) {
            x[r][k][e] = nx[r][k][e];
            g[r][k][e] = BACK ? ng[r][k][e] : 0.0f;
          }
      if (i + 1 < m.per) request(h + groups);
#pragma unroll
      for (int r = 0; r < R; ++r) {
        if (BACK) u[r].apply(g[r]);
#pragma unroll
        for (int k = 0; k < 2; ++k)
#pragma unroll
          for (int e = 0; e < V; ++e) {
            sum += x[r][k][e] * x[r][k][e];
            if (BACK) dot += w[r][k][e] * g[r][k][e] * x[r][k][e];
          }
      }
      if (norm) {
        sum = head_sum(sum, a.lanes);
        if (BACK) dot = head_sum(dot, a.lanes);
      }
      // (heads that are none would divide by 0 where eps is 0)
      const float rms = norm && on ? 1.0f / __fsqrt_rn(sum * inv_dim + a.eps) : 1.0f;
      const float back = rms * rms * (dot * inv_dim);
#pragma unroll
      for (int r = 0; r < R; ++r) {
        float o[2][V];
#pragma unroll
        for (int k = 0; k < 2; ++k)
#pragma unroll
          for (int e = 0; e < V; ++e) {
            const float v = x[r][k][e];
            if (!BACK) {
              o[k][e] = norm ? v * rms * w[r][k][e] : v;
            } else if (norm) {
              dw[r][k][e] += g[r][k][e] * v * rms;
              o[k][e] = rms * (w[r][k][e] * g[r][k][e] - v * back);
            } else {
              o[k][e] = g[r][k][e];
            }
          }
        if (!BACK) u[r].apply(o);
        if (on) {
          if (t[r].a < a.dim) store_v<V, ONCE>(m.y + at + t[r].a, o[0]);
          if (t[r].b < a.dim) store_v<V, ONCE>(m.y + at + t[r].b, o[1]);
        }
      }
    }
  }
  if constexpr (BACK) {
    if (!norm) return;
    // the groups of a wave, then the waves in order
    __shared__ float red[kWaves][kMaxDim];
    for (int d = a.lanes; d < 64; d <<= 1) {
#pragma unroll
      for (int r = 0; r < R; ++r)
#pragma unroll
        for (int k = 0; k < 2; ++k)
#pragma unroll
          for (int e = 0; e < V; ++e) dw[r][k][e] += __shfl_xor(dw[r][k][e], d);
    }
#pragma unroll
    for (int r = 0; r < R; ++r)
#pragma unroll
      for (int k = 0; k < 2; ++k)
#pragma unroll
        for (int e = 0; e < V; ++e) {
          const int at = (k == 0 ? t[r].a : t[r].b) + e;
          if (group == 0 && at < a.dim) red[wave][at] = dw[r][k][e];
        }
    __syncthreads();
    for (int i = threadIdx.x; i < a.dim; i += kThreads)
      m.part[((size_t)blockIdx.x - m.wg0) * a.dim + i] = ((red[0][i] + red[1][i]) + red[2][i]) + red[3][i];
  }
}

// The workgroups' sums, added in a fixed order: 16 columns a workgroup, each
// group of 16 threads every 64th sum, the groups one after another.
struct SumArgs {
  const float* part[kMaxInputs];
  float* out[kMaxInputs];
  int n[kMaxInputs];
  int dim;
};
__global__ __launch_bounds__(1024) void heads_sum_kernel(SumArgs a) {
  __shared__ float red[64][16];
  const int col = threadIdx.x & 15, group = threadIdx.x >> 4;
  const int i = (int)blockIdx.x * 16 + col;
  const int y = blockIdx.y;
  float sum = 0.0f;
  if (i < a.dim) {
#pragma unroll 8
    for (int q = group; q < a.n[y]; q += 64) sum += a.part[y][(size_t)q * a.dim + i];
  }
  red[group][col] = sum;
  __syncthreads();
  if (group == 0 && i < a.dim) {
    for (int w = 1; w < 64; ++w) sum += red[w][col];
    a.out[y][i] = sum;
  }
}

using namespace spdp;

// The numbers that a lane reads at once, and the lanes and workgroups that
// follow: 16 bytes where the pairs and heads divide into such vectors, else
// pairs of neighbours, else single numbers (half-split pairs of an odd half).
// Workgroups: each wave has a token's heads, or so many of them that about
// four workgroups per CU result.
struct HeadsPlan {
  int v, slots, lanes, rounds;  // rounds: slots of a lane
  int per[kMaxInputs];
  int wg0[kMaxInputs + 1];
};
void plan_heads(const spdp_heads_t* in, int inputs, const spdp_rotation_t* r, long long n_tokens, bool back, int cus, HeadsPlan* p) {
  const int half = r->rot / 2;
  if (r->interleaved ? r->dim % 16 == 0 : half % 8 == 0 && r->dim % 8 == 0)
    p->v = 8;
  else
    p->v = r->interleaved || half % 2 == 0 ? 2 : 1;
  const int lead = r->interleaved ? 0 : half / p->v;
  const int rest = r->dim - (r->interleaved ? 0 : r->rot);
  p->slots = lead + (rest + 2 * p->v - 1) / (2 * p->v);
  p->lanes = 1;
  while (p->lanes < p->slots && p->lanes < 64) p->lanes *= 2;
  p->rounds = (p->slots + 63) / 64;
  const int groups = 64 / p->lanes;
  long long all = 0, waves = 4ll * cus * kWaves;
  for (int i = 0; i < inputs; ++i) all += n_tokens * in[i].heads;
  const long long most_per = std::max<long long>(1, std::min<long long>(8, all / (groups * waves)));
  long long rounds[kMaxInputs], sum = 0;
  for (int i = 0; i < inputs; ++i) {
    // equal shares of the heads
    const long long groups_of = (in[i].heads + groups - 1) / groups;
    const long long parts = (groups_of + most_per - 1) / most_per;
    p->per[i] = (int)((groups_of + parts - 1) / parts);
    const int chunk = groups * p->per[i];
    rounds[i] = n_tokens * ((in[i].heads + chunk - 1) / chunk);
    sum += rounds[i];
  }
  // backward: each workgroup's share of the weights' gradient is reduced, written
  // and read again: as many as a CU's registers hold (2 / 3 / 4 per CU: 2048
  // tokens, 40 + 8 heads of 96, 26 / 21 / 23 us; 512, 64 + 8 of 128, 15 / 14 / 18;
  // 4096, 32 + 8 of 128, 35 / 31 / 29)
  const long long most = back ? 3ll * cus : 1ll << 22;
  p->wg0[0] = 0;
  for (int i = 0; i < inputs; ++i) {
    const long long want = (rounds[i] + kWaves - 1) / kWaves;
    p->wg0[i + 1] = p->wg0[i] + (int)std::max<long long>(1, std::min(want, most * rounds[i] / std::max<long long>(1, sum)));
  }
}

int check(const spdp_heads_t* in, int32_t inputs, const spdp_rotation_t* r, int64_t n_tokens) {
  if (!in || !r) return fail(SPDP_ERR_INVALID_ARG, "inputs or rotation is NULL");
  if (inputs < 1 || inputs > kMaxInputs) return fail(SPDP_ERR_INVALID_ARG, "the number of inputs must lie in [1, 8]");
  if (!r->positions || !r->cosine || !r->sine) return fail(SPDP_ERR_INVALID_ARG, "positions, cosine or sine is NULL");
  if (n_tokens < 1 || r->table < 1) return fail(SPDP_ERR_INVALID_ARG, "n_tokens and table must be at least 1");
  if (n_tokens > 1 << 24 || r->table > 1 << 30) return fail(SPDP_ERR_UNSUPPORTED, "more than 2^24 tokens or 2^30 positions");
  if (r->dim < 2 || r->rot < 2 || r->dim % 2 || r->rot % 2 || r->rot > r->dim)
    return fail(SPDP_ERR_INVALID_ARG, "dim and rot must be even, with 2 <= rot <= dim");
  if (r->dim > kMaxDim) return fail(SPDP_ERR_UNSUPPORTED, "heads of more than 512 numbers");
  if (!(r->eps >= 0.0f) || r->eps > 1e30f) return fail(SPDP_ERR_INVALID_ARG, "eps must be >= 0 and finite");
  for (int i = 0; i < inputs; ++i) {
    if (!in[i].x) return fail(SPDP_ERR_INVALID_ARG, "x is NULL");
    if (in[i].heads < 1) return fail(SPDP_ERR_INVALID_ARG, "heads must be at least 1");
    if (in[i].heads > 65536) return fail(SPDP_ERR_UNSUPPORTED, "more than 65536 heads");
  }
  return SPDP_OK;
}

template <int V, int R, bool PAIRS, bool ONCE>
void launch(const HeadsArgs& a, bool back, dim3 grid, hipStream_t s) {
  if (back)
    hipLaunchKernelGGL((heads_kernel<V, R, PAIRS, true, ONCE>), grid, dim3(kThreads), 0, s, a);
  else
    hipLaunchKernelGGL((heads_kernel<V, R, PAIRS, false, ONCE>), grid, dim3(kThreads), 0, s, a);
}
template <int V, int R, bool ONCE>
void launch_pairs(const HeadsArgs& a, bool pairs, bool back, dim3 grid, hipStream_t s) {
  if constexpr (V > 1)
    if (pairs) return launch<V, R, true, ONCE>(a, back, grid, s);
  launch<V, R, false, ONCE>(a, back, grid, s);
}

size_t grad_bytes(const spdp_heads_t* in, int inputs, int dim, const HeadsPlan& p) {
  size_t bytes = 0;
  for (int i = 0; i < inputs; ++i)
    if (in[i].weight) bytes += aligned((size_t)(p.wg0[i + 1] - p.wg0[i]) * dim * 4);
  return bytes;
}

int heads(const spdp_heads_t* in, int32_t inputs, const spdp_rotation_t* r, int64_t n_tokens, bool back, void* workspace,
          size_t workspace_bytes, void* stream) {
  int st = check(in, inputs, r, n_tokens);
  if (st != SPDP_OK) return st;
  // an output may be its own input as a whole, and overlaps nothing else
  for (int i = 0; i < inputs; ++i) {
    if (!in[i].y) return fail(SPDP_ERR_INVALID_ARG, "y is NULL");
    if (back && !in[i].dy) return fail(SPDP_ERR_INVALID_ARG, "dy is NULL");
    if (back && (in[i].weight != nullptr) != (in[i].dweight != nullptr))
      return fail(SPDP_ERR_INVALID_ARG, "dweight goes with weight");
    const size_t row = (size_t)n_tokens * r->dim * 2, n = row * in[i].heads;
    for (int j = 0; j < inputs; ++j) {
      const size_t other = row * in[j].heads;
      if (overlap(in[i].y, n, in[j].x, other) && !(i == j && in[i].y == in[j].x))
        return fail(SPDP_ERR_INVALID_ARG, "an output overlaps an input");
      if (back && overlap(in[i].y, n, in[j].dy, other) && !(i == j && in[i].y == in[j].dy))
        return fail(SPDP_ERR_INVALID_ARG, "an output overlaps an input");
      if (i != j && overlap(in[i].y, n, in[j].y, other)) return fail(SPDP_ERR_INVALID_ARG, "outputs overlap");
      if (overlap(in[i].y, n, in[j].weight, (size_t)r->dim * 2)) return fail(SPDP_ERR_INVALID_ARG, "an output overlaps a weight");
    }
    const size_t table = (size_t)r->table * r->rot * 2;
    if (back && in[i].dweight) {
      const size_t own = (size_t)r->dim * 4;
      if (overlap(in[i].dweight, own, r->positions, (size_t)n_tokens * 4) || overlap(in[i].dweight, own, r->cosine, table) ||
          overlap(in[i].dweight, own, r->sine, table))
        return fail(SPDP_ERR_INVALID_ARG, "a weight's gradient overlaps the positions or the tables");
      for (int j = 0; j < inputs; ++j) {
        const size_t other = row * in[j].heads;
        if (overlap(in[i].dweight, own, in[j].x, other) || overlap(in[i].dweight, own, in[j].dy, other) ||
            overlap(in[i].dweight, own, in[j].y, other) || overlap(in[i].dweight, own, in[j].weight, (size_t)r->dim * 2) ||
            (i != j && overlap(in[i].dweight, own, in[j].dweight, own)))
          return fail(SPDP_ERR_INVALID_ARG, "a weight's gradient overlaps another array");
      }
    }
    if (overlap(in[i].y, n, r->positions, (size_t)n_tokens * 4) || overlap(in[i].y, n, r->cosine, table) ||
        overlap(in[i].y, n, r->sine, table))
      return fail(SPDP_ERR_INVALID_ARG, "an output overlaps the positions or the tables");
  }
  int cus = 1;
  st = compute_units(&cus);
  if (st != SPDP_OK) return st;
  HeadsPlan p;
  plan_heads(in, inputs, r, n_tokens, back, cus, &p);
  HeadsArgs a;
  std::memset(&a, 0, sizeof(a));
  SumArgs sum;
  std::memset(&sum, 0, sizeof(sum));
  sum.dim = r->dim;
  int sums = 0;
  if (back) {
    st = check_workspace(workspace, workspace_bytes, grad_bytes(in, inputs, r->dim, p));
    if (st != SPDP_OK) return st;
  }
  unsigned char* ws = static_cast<unsigned char*>(workspace);
  size_t bytes = 0;
  for (int i = 0; i < inputs; ++i) {
    bytes += (size_t)n_tokens * in[i].heads * r->dim * 2;
    a.m[i] = HeadsInput{in[i].x, in[i].weight, in[i].dy, in[i].y, nullptr, in[i].heads, p.wg0[i], p.per[i]};
    if (back && in[i].weight) {
      const int wgs = p.wg0[i + 1] - p.wg0[i];
      a.m[i].part = reinterpret_cast<float*>(ws);
      sum.part[sums] = a.m[i].part;
      sum.out[sums] = in[i].dweight;
      sum.n[sums++] = wgs;
      ws += aligned((size_t)wgs * r->dim * 4);
    }
  }
  a.pos = r->positions;
  a.cosine = r->cosine;
  a.sine = r->sine;
  a.eps = r->eps;
  a.inputs = inputs;
  a.n_tokens = (int)n_tokens;
  a.positions = (int)r->table;
  a.dim = r->dim;
  a.half = r->rot / 2;
  const bool pairs = r->interleaved != 0;
  a.lanes = p.lanes;
  const dim3 grid((unsigned)p.wg0[inputs]);
  auto s = static_cast<hipStream_t>(stream);
  // Outputs larger than the L2 caches (4 MB on each of 8 dies) go past them, and the
  // backward pass's inputs, which nothing reads afterwards (through / past them:
  // 4096 tokens of 32 + 32 heads of 128 31.3 / 24.8 us, backward 51.6 / 46.4; 2048 of
  // 40 + 8 of 96, which fit, 10.3 / 13.2, 20.3 / 22.2)
  const bool once = bytes > (size_t)32 << 20;
  if (p.v == 8 && once)
    launch_pairs<8, 1, true>(a, pairs, back, grid, s);
  else if (p.v == 8)
    launch_pairs<8, 1, false>(a, pairs, back, grid, s);
  else if (p.v == 2 && p.rounds == 1)
    launch_pairs<2, 1, false>(a, pairs, back, grid, s);
  else if (p.v == 2)
    launch_pairs<2, 2, false>(a, pairs, back, grid, s);
  else
    launch_pairs<1, 4, false>(a, pairs, back, grid, s);
  hipError_t e = hipGetLastError();
  if (e == hipSuccess && sums > 0) {
    hipLaunchKernelGGL(heads_sum_kernel, dim3((unsigned)((r->dim + 15) / 16), (unsigned)sums), dim3(1024), 0, s, sum);
    e = hipGetLastError();
  }
  return e == hipSuccess ? SPDP_OK : hip_fail(e, "kernel launch");
}

}  // namespace

extern "C" {

int spdp_rotate_heads(const spdp_heads_t* inputs, int32_t n_inputs, const spdp_rotation_t* rotation, int64_t n_tokens,
                      void* stream) {
  return guarded([&] { return heads(inputs, n_inputs, rotation, n_tokens, false, nullptr, 0, stream); });
}

int spdp_rotate_heads_grad_workspace(const spdp_heads_t* inputs, int32_t n_inputs, const spdp_rotation_t* rotation,
                                     int64_t n_tokens, size_t* bytes) {
  return guarded([&] {
    if (!bytes) return fail(SPDP_ERR_INVALID_ARG, "bytes is NULL");
    int st = check(inputs, n_inputs, rotation, n_tokens);
    int cus = 1;
    if (st == SPDP_OK) st = compute_units(&cus);
    if (st != SPDP_OK) return st;
    HeadsPlan p;
    plan_heads(inputs, n_inputs, rotation, n_tokens, true, cus, &p);
    *bytes = grad_bytes(inputs, n_inputs, rotation->dim, p);
    return (int)SPDP_OK;
  });
}

int spdp_rotate_heads_grad(const spdp_heads_t* inputs, int32_t n_inputs, const spdp_rotation_t* rotation,
                           int64_t n_tokens, void* workspace, size_t workspace_bytes, void* stream) {
  return guarded([&] { return heads(inputs, n_inputs, rotation, n_tokens, true, workspace, workspace_bytes, stream); });
}

}  // extern "C"
