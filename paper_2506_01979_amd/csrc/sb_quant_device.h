// Rows of activations to 8-bit codes, shared by the kernels that produce them.
#pragma once

#include "sb_device.h"

namespace sb {

// The 8-bit operand of a projection: [row / 16][k / 64][lane][16], fragments of
// 1 KB in the order of the 16x16x64 integer matrix instruction: lane l holds
// row l % 16, columns 16 (l / 16) .. + 15 of the k-step.  An "item" is 16
// consecutive columns of a row, one lane's bytes.
__device__ __forceinline__ size_t item_offset(int row, int item, int ks) {
  return ((((size_t)(row >> 4) * ks + (item >> 2)) * 64) + (item & 3) * 16 + (row & 15)) * 16;
}

// Sixteen values to codes: nearest(127 x / amax), ties to even, one IEEE
// division each (live: amax is positive and finite; otherwise zeros).  From amax =
// 2^100 on, where 127 x may pass float32, x and amax are taken at 2^-16: the
// same quotients but for values below 2^-200 of amax, code 0.
__device__ __forceinline__ uint4 codes16(const float (&x)[16], float amax, bool live) {
  const float down = amax >= 0x1p100f ? 0x1p-16f : 1.0f;
  const float num = 127.0f * down, den = amax * down;
  uint32_t w[4];
#pragma unroll
  for (int j = 0; j < 4; ++j) {
    w[j] = 0;
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      const int q = live ? (int)rintf(x[4 * j + e] * num / den) : 0;
      w[j] |= (uint32_t)(q & 0xff) << (8 * e);
    }
  }
  return make_uint4(w[0], w[1], w[2], w[3]);
}

// A row of a workgroup of NT threads, IPT items per thread (item threadIdx.x + j
// NT), to codes and its scale amax / 127 times mul.  The largest magnitude is
// found on the bit patterns, where NaN and infinity are the largest: they make
// the scale NaN.  red: NT / 64 words of LDS, free on entry.
template <int NT, int IPT>
__device__ __forceinline__ void quantize_row(const float (&x)[IPT][16], int row, int ks, float mul,
                                             uint8_t *codes, float *scale, uint32_t *red) {
  uint32_t top = 0;
#pragma unroll
  for (int j = 0; j < IPT; ++j)
#pragma unroll
    for (int e = 0; e < 16; ++e) top = max(top, __float_as_uint(x[j][e]) & 0x7fffffffu);
  for (int o = 32; o > 0; o >>= 1) top = max(top, (uint32_t)__shfl_xor((int)top, o, 64));
  if ((threadIdx.x & 63) == 0) red[threadIdx.x >> 6] = top;
  __syncthreads();
  top = red[0];
#pragma unroll
  for (int i = 1; i < NT / 64; ++i) top = max(top, red[i]);
  const bool finite = top < 0x7f800000u;
  const float amax = __uint_as_float(top);
  if (threadIdx.x == 0) scale[row] = finite ? amax / 127.0f * mul : NAN;
#pragma unroll
  for (int j = 0; j < IPT; ++j) {
    const int item = threadIdx.x + j * NT;
    if (item < ks * 4)
      *(uint4 *)(codes + item_offset(row, item, ks)) = codes16(x[j], amax, finite && top != 0);
  }
}

}  // namespace sb
