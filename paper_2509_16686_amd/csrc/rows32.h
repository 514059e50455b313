// What the attention kernels of 32 query rows a wave share: the layout of a key
// tile in LDS (key_tile.h), and lane operations on the accumulators of v_mfma_f32_32x32x16.
#pragma once

#include "device_common.h"
#include "key_tile.h"

namespace egmla {

typedef __attribute__((ext_vector_type(16))) float px_f32x16_t;

// Holds a block of accumulators in accumulation or ordinary registers at this point.
__device__ __forceinline__ void in_agprs(px_f32x16_t& x) { asm volatile("" : "+a"(x)); }
__device__ __forceinline__ void in_vgprs(px_f32x16_t& x) { asm volatile("" : "+v"(x)); }

// Maximum and sum of lanes i and i ^ 32, the same value (same order) in both.
__device__ __forceinline__ float half_max(float x) {
  const uint32_t u = __float_as_uint(x);
  const auto s = __builtin_amdgcn_permlane32_swap(u, u, false, false);
  return fmaxf(__uint_as_float(s[0]), __uint_as_float(s[1]));
}
__device__ __forceinline__ float half_sum(float x) {
  const uint32_t u = __float_as_uint(x);
  const auto s = __builtin_amdgcn_permlane32_swap(u, u, false, false);
  return __uint_as_float(s[0]) + __uint_as_float(s[1]);
}

}  // namespace egmla
