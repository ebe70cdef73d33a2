// Device helpers shared by the attention kernels.
#pragma once

#include "sb_device.h"

namespace sb {

// Workgroup barrier for LDS traffic only (does not wait for global loads).
__device__ __forceinline__ void lds_barrier() {
  asm volatile("s_waitcnt lgkmcnt(0)\n\ts_barrier" ::: "memory");
}

// Two floats to packed bf16 (round to nearest even), one instruction.
__device__ __forceinline__ uint32_t pack_bf16x2(float lo, float hi) {
  typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
  typedef float f32x2 __attribute__((ext_vector_type(2)));
  const f32x2 v = {lo, hi};
  return __builtin_bit_cast(uint32_t, __builtin_convertvector(v, bf16x2));
}

// Max / sum over the lane pairs (l, l ^ 16) and (l, l ^ 32) with the gfx950
// lane-swap instructions: swapping a value with itself yields, in every lane,
// the pair's even-row and odd-row values.
__device__ __forceinline__ float max_x16(float v) {
  const auto r = __builtin_amdgcn_permlane16_swap(__builtin_bit_cast(uint32_t, v),
                                                  __builtin_bit_cast(uint32_t, v), false, false);
  return fmaxf(__builtin_bit_cast(float, (uint32_t)r[0]), __builtin_bit_cast(float, (uint32_t)r[1]));
}
__device__ __forceinline__ float max_x32(float v) {
  const auto r = __builtin_amdgcn_permlane32_swap(__builtin_bit_cast(uint32_t, v),
                                                  __builtin_bit_cast(uint32_t, v), false, false);
  return fmaxf(__builtin_bit_cast(float, (uint32_t)r[0]), __builtin_bit_cast(float, (uint32_t)r[1]));
}
__device__ __forceinline__ float sum_x16(float v) {
  const auto r = __builtin_amdgcn_permlane16_swap(__builtin_bit_cast(uint32_t, v),
                                                  __builtin_bit_cast(uint32_t, v), false, false);
  return __builtin_bit_cast(float, (uint32_t)r[0]) + __builtin_bit_cast(float, (uint32_t)r[1]);
}
__device__ __forceinline__ float sum_x32(float v) {
  const auto r = __builtin_amdgcn_permlane32_swap(__builtin_bit_cast(uint32_t, v),
                                                  __builtin_bit_cast(uint32_t, v), false, false);
  return __builtin_bit_cast(float, (uint32_t)r[0]) + __builtin_bit_cast(float, (uint32_t)r[1]);
}

// Visibility of the 8 keys k0 .. k0 + 7 (k0 a multiple of 8) for a row with
// ancestor mask anc (LDS): prefix slots are visible, tree slot kv_len + j is
// visible when bit j is set, slots >= nkeys are not.
__device__ __forceinline__ uint32_t visible8(const uint32_t *anc, int k0, int kv_len, int nkeys) {
  uint32_t vis;
  const int jt = k0 - kv_len;
  if (jt + 8 <= 0) {
    vis = 0xffu;
  } else if (jt >= 0) {
    const int wi = jt >> 5, sh = jt & 31;  // bits jt .. jt + 7 of the 256-bit mask
    const uint64_t win = (uint64_t)anc[wi] | ((uint64_t)(wi < 7 ? anc[wi + 1] : 0u) << 32);
    vis = (uint32_t)(win >> sh) & 0xffu;
  } else {
    const int pre = -jt;  // 1..7 prefix keys, then tree bits 0 ..
    vis = ((anc[0] << pre) | ((1u << pre) - 1u)) & 0xffu;
  }
  const int valid = nkeys - k0;
  if (valid < 8) vis &= valid > 0 ? (1u << valid) - 1u : 0u;
  return vis;
}

}  // namespace sb
