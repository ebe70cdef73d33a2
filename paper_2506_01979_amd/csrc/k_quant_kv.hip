// Blocks of the prefix cache to 8 bits and back, and the move of what a
// commit leaves in the tail.
//
// A block is 64 tokens x head_dim of one (layer, KV head), of K or V:
//   amax = max |x|, scale = fl32(amax / top), code = nearest(x top / amax),
//   top = 127 (int8) or 448 (e4m3).
// x has 8 significant bits and top at most 7, so x top is exact in float32 (of a
// block with amax >= 2^100, whose x top may pass float32, x and amax are taken at
// 2^-16: values that this rounds are below 2^-200 of amax, code 0), and
// one IEEE division gives the code of the formula: the quotient of two such
// numbers either is a tie of the 8-bit type exactly (and then a float32) or
// lies at least 2^-17 of its size away from one, far outside the division's
// rounding.  The largest magnitude is found on the bit patterns, where NaN and
// infinity are the largest.
//
// One workgroup per block and matrix; a thread loads the values of the 16
// codes it stores (two 16-byte loads each), all before the first use.  Bound by
// HBM: 32 layers x 32 heads x 4 blocks of 64 x 128 take 54 us to quantise and
// 32 to read back, 403 MB in all at 4.7 TB/s; ten times as many, 5.1 TB/s.
#include <math.h>

#include "sb_device.h"
#include "sb_internal_fwd.h"

namespace sb {
namespace {

constexpr int kT = 256;

// Where fragment item i (fragment i / 64, lane i % 64) of a block has its two
// halves of 8 values in the 16-bit cache: element offsets from the head's
// first slot, K [slot][D], V [D][cap].
template <int D>
__device__ __forceinline__ void item_at(int i, bool is_v, int slot, int cap, size_t (&at)[2]) {
  const int c = i >> 6, lr = i & 15, lg = (i >> 4) & 3;
  if (is_v) {
    at[0] = (size_t)(16 * c + lr) * cap + slot + 8 * lg;
    at[1] = at[0] + 32;
  } else {
    const int kt = c / (D / 64), p = c % (D / 64);
    const int key = 32 * (kt >> 1) + 8 * (lr >> 2) + 4 * (kt & 1) + (lr & 3);
    at[0] = (size_t)(slot + key) * D + 64 * p + 8 * lg;
    at[1] = at[0] + 32;
  }
}

template <int D, int FMT>
__global__ __launch_bounds__(kT) void k_kv_quantize(QuantKvArgs a) {
  constexpr int IPT = D * 4 / kT;  // items per thread
  __shared__ uint32_t smax[kT / 64];
  const bool is_v = blockIdx.y != 0;
  const int head = blockIdx.x / a.n_blocks, b = blockIdx.x % a.n_blocks;
  const uint16_t *src = (is_v ? a.v16 : a.k16) + (size_t)head * a.cap * D;
  uint4 x[IPT][2];
#pragma unroll
  for (int j = 0; j < IPT; ++j) {
    size_t at[2];
    item_at<D>(threadIdx.x + j * kT, is_v, a.slot + b * SB_KV_BLOCK, a.cap, at);
    x[j][0] = *(const uint4 *)(src + at[0]);
    x[j][1] = *(const uint4 *)(src + at[1]);
  }
  uint32_t top = 0;
#pragma unroll
  for (int j = 0; j < IPT; ++j)
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      const uint32_t w[4] = {x[j][h].x, x[j][h].y, x[j][h].z, x[j][h].w};
#pragma unroll
      for (int e = 0; e < 4; ++e) top = max(top, max(w[e] & 0x7fffu, (w[e] >> 16) & 0x7fffu));
    }
  for (int o = 32; o > 0; o >>= 1) top = max(top, (uint32_t)__shfl_xor((int)top, o, 64));
  if ((threadIdx.x & 63) == 0) smax[threadIdx.x >> 6] = top;
  __syncthreads();
  top = max(max(smax[0], smax[1]), max(smax[2], smax[3]));
  const bool finite = top < 0x7f80u;
  const float amax = __uint_as_float(top << 16);
  constexpr float kTop = FMT == SB_KV_INT8 ? 127.0f : 448.0f;
  const size_t block = (size_t)head * a.cap_blocks + a.block + b;
  if (threadIdx.x == 0) (is_v ? a.v_scale : a.k_scale)[block] = finite ? amax / kTop : NAN;
  const bool codes = finite && top != 0;
  const float down = amax >= 0x1p100f ? 0x1p-16f : 1.0f;
  const float num = kTop * down, den = amax * down;
  uint8_t *dst = (is_v ? a.v : a.k) + block * (SB_KV_BLOCK * D);
#pragma unroll
  for (int j = 0; j < IPT; ++j) {
    uint32_t out[4];
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      const uint32_t w[4] = {x[j][h].x, x[j][h].y, x[j][h].z, x[j][h].w};
      float y[8];
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        const float v = bf2f((uint16_t)(w[e >> 1] >> (16 * (e & 1))));
        y[e] = codes ? v * num / den : 0.0f;
      }
#pragma unroll
      for (int e = 0; e < 2; ++e) {
        uint32_t r = 0;
        if (FMT == SB_KV_INT8) {
#pragma unroll
          for (int i = 0; i < 4; ++i) r |= (uint32_t)((int)rintf(y[4 * e + i]) + 128) << (8 * i);
        } else {
          r = (uint32_t)__builtin_amdgcn_cvt_pk_fp8_f32(y[4 * e], y[4 * e + 1], 0, false);
          r = (uint32_t)__builtin_amdgcn_cvt_pk_fp8_f32(y[4 * e + 2], y[4 * e + 3], (int)r, true);
        }
        out[2 * h + e] = r;
      }
    }
    ((uint4 *)dst)[threadIdx.x + j * kT] = make_uint4(out[0], out[1], out[2], out[3]);
  }
}

template <int D, int FMT>
__global__ __launch_bounds__(kT) void k_kv_dequantize(QuantKvArgs a) {
  constexpr int IPT = D * 4 / kT;
  const bool is_v = blockIdx.y != 0;
  const int head = blockIdx.x / a.n_blocks, b = blockIdx.x % a.n_blocks;
  const size_t block = (size_t)head * a.cap_blocks + a.block + b;
  const uint8_t *src = (is_v ? a.v : a.k) + block * (SB_KV_BLOCK * D);
  uint16_t *dst = (is_v ? a.v16 : a.k16) + (size_t)head * a.cap * D;
  const float scale = (is_v ? a.v_scale : a.k_scale)[block];
  uint4 x[IPT];
#pragma unroll
  for (int j = 0; j < IPT; ++j) x[j] = ((const uint4 *)src)[threadIdx.x + j * kT];
#pragma unroll
  for (int j = 0; j < IPT; ++j) {
    size_t at[2];
    item_at<D>(threadIdx.x + j * kT, is_v, a.slot + b * SB_KV_BLOCK, a.cap, at);
    const uint32_t w[4] = {x[j].x, x[j].y, x[j].z, x[j].w};
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      float y[8];
#pragma unroll
      for (int e = 0; e < 2; ++e) {
        const uint32_t r = w[2 * h + e];
        if (FMT == SB_KV_INT8) {
#pragma unroll
          for (int i = 0; i < 4; ++i) y[4 * e + i] = (float)((int)((r >> (8 * i)) & 0xffu) - 128);
        } else {
          y[4 * e + 0] = __builtin_amdgcn_cvt_f32_fp8((int)r, 0);
          y[4 * e + 1] = __builtin_amdgcn_cvt_f32_fp8((int)r, 1);
          y[4 * e + 2] = __builtin_amdgcn_cvt_f32_fp8((int)r, 2);
          y[4 * e + 3] = __builtin_amdgcn_cvt_f32_fp8((int)r, 3);
        }
      }
      uint4 o;
      o.x = f2bf(y[0] * scale) | ((uint32_t)f2bf(y[1] * scale) << 16);
      o.y = f2bf(y[2] * scale) | ((uint32_t)f2bf(y[3] * scale) << 16);
      o.z = f2bf(y[4] * scale) | ((uint32_t)f2bf(y[5] * scale) << 16);
      o.w = f2bf(y[6] * scale) | ((uint32_t)f2bf(y[7] * scale) << 16);
      *(uint4 *)(dst + at[h]) = o;
    }
  }
}

// One workgroup per (layer, KV head): n < 64 rows of K, and n elements of
// every V row, from slot `from` >= 64 to slot 0, so no source is overwritten.
__global__ __launch_bounds__(kT) void k_kv_move(uint16_t *__restrict__ k, uint16_t *__restrict__ v,
                                                int cap, int d, int from, int n) {
  uint16_t *kh = k + (size_t)blockIdx.x * cap * d, *vh = v + (size_t)blockIdx.x * cap * d;
  for (int i = threadIdx.x; i < n * (d / 8); i += kT)
    ((uint4 *)kh)[i] = ((const uint4 *)(kh + (size_t)from * d))[i];
  for (int i = threadIdx.x; i < d * 8; i += kT) {
    uint16_t *row = vh + (size_t)(i >> 3) * cap;
    const int j = (i & 7) * 8;
    if (j + 8 <= n) {
      *(uint4 *)(row + j) = *(const uint4 *)(row + from + j);
    } else {
      for (int e = j; e < n; ++e) row[e] = row[from + e];
    }
  }
}

template <template <int, int> class F>
hipError_t dispatch(const QuantKvArgs &a, hipStream_t s) {
  if (a.head_dim == 128)
    return a.format == SB_KV_INT8 ? F<128, SB_KV_INT8>::launch(a, s) : F<128, SB_KV_E4M3>::launch(a, s);
  if (a.head_dim == 64)
    return a.format == SB_KV_INT8 ? F<64, SB_KV_INT8>::launch(a, s) : F<64, SB_KV_E4M3>::launch(a, s);
  return hipErrorInvalidValue;
}
template <int D, int FMT>
struct Quantize {
  static hipError_t launch(const QuantKvArgs &a, hipStream_t s) {
    hipLaunchKernelGGL((k_kv_quantize<D, FMT>), dim3(a.heads * a.n_blocks, 2), dim3(kT), 0, s, a);
    return hipGetLastError();
  }
};
template <int D, int FMT>
struct Dequantize {
  static hipError_t launch(const QuantKvArgs &a, hipStream_t s) {
    hipLaunchKernelGGL((k_kv_dequantize<D, FMT>), dim3(a.heads * a.n_blocks, 2), dim3(kT), 0, s, a);
    return hipGetLastError();
  }
};

}  // namespace

hipError_t launch_kv_quantize(const QuantKvArgs &a, hipStream_t s) { return dispatch<Quantize>(a, s); }
hipError_t launch_kv_dequantize(const QuantKvArgs &a, hipStream_t s) {
  return dispatch<Dequantize>(a, s);
}
hipError_t launch_kv_move(uint16_t *k, uint16_t *v, int heads, int cap, int head_dim, int from,
                          int n, hipStream_t s) {
  hipLaunchKernelGGL(k_kv_move, dim3(heads), dim3(kT), 0, s, k, v, cap, head_dim, from, n);
  return hipGetLastError();
}

}  // namespace sb
