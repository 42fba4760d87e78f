// Loads and LDS reads of a lane, shared by the kernels beside the pruned
// products.
#pragma once

#include "expand.h"

namespace spdp_dev {

typedef _Float16 half4 __attribute__((ext_vector_type(4)));
typedef short short4v __attribute__((ext_vector_type(4)));

// orders a wave's own LDS accesses across its lanes
__device__ __forceinline__ void wave_fence() { __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront"); }

// eight fp16 from p (any alignment)
__device__ __forceinline__ half8 load8(const uint16_t* p) {
  half8 v;
  __builtin_memcpy(&v, p, 16);
  return v;
}
// p[0 .. n - 1], then zeros
__device__ __forceinline__ half8 load_upto8(const uint16_t* p, int n) {
  half8 v;
#pragma unroll
  for (int e = 0; e < 8; ++e) v[e] = e < n ? __builtin_bit_cast(_Float16, p[e]) : (_Float16)0;
  return v;
}
// v[0 .. min(n, 8) - 1] to p (any alignment)
__device__ __forceinline__ void store8_inside(uint16_t* p, half8 v, int n) {
  if (n >= 8) {
    __builtin_memcpy(p, &v, 16);
    return;
  }
#pragma unroll
  for (int e = 0; e < 8; ++e) {
    const _Float16 h = v[e];  // (a bit cast of v[e] itself is one of v[0])
    if (e < n) p[e] = __builtin_bit_cast(uint16_t, h);
  }
}
__device__ __forceinline__ half8 load8_inside(const uint16_t* p, int n) { return n >= 8 ? load8(p) : load_upto8(p, n); }

// the same of data that is larger than the caches and read once
__device__ __forceinline__ half8 load8_once(const uint16_t* p, int n) {
  typedef half8 half8_any __attribute__((aligned(2)));
  return n >= 8 ? __builtin_nontemporal_load(reinterpret_cast<const half8_any*>(p)) : load_upto8(p, n);
}

// lane's operand of the 32 columns from `col` on and the eight rows from `row`
// + 8 (lane / 32) on, of a row-major fp16 tile in LDS of `stride` bytes a row.
// Each group of 16 lanes reads 4 rows x 16 columns: lane i supplies the address
// of row i / 4, columns 4 (i mod 4) .. + 3, and gets column i of the four rows.
__device__ __forceinline__ half8 read_transposed(const unsigned char* tile, int stride, int row, int col) {
  const int lane = threadIdx.x & 63;
  const int i = lane & 15;
  const uint32_t p =
      lds_addr(tile) + (uint32_t)((row + 8 * (lane >> 5) + (i >> 2)) * stride + 2 * (col + (lane & 16) + 4 * (i & 3)));
  typedef __attribute__((address_space(3))) short4v* lds4;
  const half4 a = __builtin_bit_cast(half4, __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds4)(uintptr_t)p));
  const half4 b = __builtin_bit_cast(half4, __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds4)(uintptr_t)(p + 4u * (uint32_t)stride)));
  return half8{a[0], a[1], a[2], a[3], b[0], b[1], b[2], b[3]};
}

}  // namespace spdp_dev
