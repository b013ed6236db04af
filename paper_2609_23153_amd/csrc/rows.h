// Device helpers of the kernels that stream rows and pages.
#pragma once

#include "common.h"

namespace sa {

// 16 bytes of data that is read once: the load does not push out what the caches
// hold (one token over a long cache: 5.5 -> 6.2 TB/s).
__device__ __forceinline__ u32x4 ld16_once(const void* p) {
  return __builtin_nontemporal_load(reinterpret_cast<const u32x4*>(p));
}

// x summed over the lane's row of 16 lanes, in each of them (DPP rotations).
__device__ __forceinline__ float row_sum_f32(float x) {
#define SA_ROR(n)                                                                              \
  x += __uint_as_float((uint32_t)__builtin_amdgcn_update_dpp(0, (int)__float_as_uint(x), 0x120 + n, \
                                                             0xF, 0xF, false))
  SA_ROR(8);
  SA_ROR(4);
  SA_ROR(2);
  SA_ROR(1);
#undef SA_ROR
  return x;
}
// x summed over the lanes of one place in the wave's four rows.
__device__ __forceinline__ float across_rows_f32(float x) {
  const uint32_t u = __float_as_uint(x);
  const auto p = __builtin_amdgcn_permlane16_swap(u, u, false, false);
  x = __uint_as_float(p[0]) + __uint_as_float(p[1]);
  const uint32_t v = __float_as_uint(x);
  const auto q = __builtin_amdgcn_permlane32_swap(v, v, false, false);
  return __uint_as_float(q[0]) + __uint_as_float(q[1]);
}
// x summed over the wave, in every lane (as wave_sum_u32).
__device__ __forceinline__ float wave_sum_f32(float x) { return across_rows_f32(row_sum_f32(x)); }

}  // namespace sa
