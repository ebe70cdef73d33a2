// What stands between the projections of an int8 model: RMSNorm, RoPE with the
// cache writes, and SwiGLU, each producing what the next launch reads.
//
// The norm keeps the factored form RMSNorm(h) g = r (h g): the codes are those
// of h g, and r goes into the row's scale.
//
// Bound by the launch and one row's way through a workgroup (7B, 33 rows: norm
// 5.6 us, RoPE and stores 4.3, SwiGLU 6.6 for 2.9 MB in).
#include <math.h>

#include "sb_internal_fwd.h"
#include "sb_quant_device.h"

namespace sb {
namespace {

constexpr int kRowT = 512;

// One workgroup per row, the row in registers; every load before the first
// use.  Columns past hidden and rows past n_tok read zeros.
template <int IPT>
__global__ __launch_bounds__(kRowT) void k_norm_quant(float *__restrict__ h,
                                                      const float *__restrict__ delta,
                                                      const float *__restrict__ g, int hidden,
                                                      int ks, int n_tok, float eps, uint8_t *codes,
                                                      float *scale, float *__restrict__ tap,
                                                      int tap_normed) {
  __shared__ float red[kRowT / 64];
  __shared__ uint32_t redq[kRowT / 64];
  const int t = blockIdx.x;
  const bool live = t < n_tok;
  const int row_bytes = hidden * 4, here = live ? row_bytes : 0;
  const __amdgpu_buffer_rsrc_t hrs = uniform_rsrc(h + (size_t)(live ? t : 0) * hidden, here);
  const __amdgpu_buffer_rsrc_t drs = uniform_rsrc(
      delta ? delta + (size_t)(live ? t : 0) * hidden : h, delta ? here : 0);
  const __amdgpu_buffer_rsrc_t grs = uniform_rsrc(g, row_bytes);
  float x[IPT][16], gv[IPT][16];
#pragma unroll
  for (int j = 0; j < IPT; ++j)
#pragma unroll
    for (int q = 0; q < 4; ++q) {
      const int c = (threadIdx.x + j * kRowT) * 16 + 4 * q;
      const int vo = c < hidden ? c * 4 : row_bytes;
      const f32x4 a = __builtin_bit_cast(f32x4, __builtin_amdgcn_raw_buffer_load_b128(hrs, vo, 0, 0));
      const f32x4 d = __builtin_bit_cast(f32x4, __builtin_amdgcn_raw_buffer_load_b128(drs, vo, 0, 0));
      const f32x4 w = __builtin_bit_cast(f32x4, __builtin_amdgcn_raw_buffer_load_b128(grs, vo, 0, 0));
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        x[j][4 * q + e] = a[e] + d[e];
        gv[j][4 * q + e] = w[e];
      }
    }
  float ss = 0.0f;
#pragma unroll
  for (int j = 0; j < IPT; ++j) {
    const int c0 = (threadIdx.x + j * kRowT) * 16;
#pragma unroll
    for (int q = 0; q < 4; ++q) {
      const f32x4 v = {x[j][4 * q], x[j][4 * q + 1], x[j][4 * q + 2], x[j][4 * q + 3]};
      if (live && c0 + 4 * q < hidden) {  // hidden is a multiple of 8
        if (delta) *(f32x4 *)(h + (size_t)t * hidden + c0 + 4 * q) = v;
        if (tap && !tap_normed) *(f32x4 *)(tap + (size_t)t * hidden + c0 + 4 * q) = v;
      }
    }
#pragma unroll
    for (int e = 0; e < 16; ++e) ss += x[j][e] * x[j][e];
  }
  for (int o = 32; o > 0; o >>= 1) ss += __shfl_xor(ss, o, 64);
  if ((threadIdx.x & 63) == 0) red[threadIdx.x >> 6] = ss;
  __syncthreads();
  ss = red[0];
#pragma unroll
  for (int i = 1; i < kRowT / 64; ++i) ss += red[i];
  const float r = live ? 1.0f / sqrtf(ss / (float)hidden + eps) : 0.0f;
#pragma unroll
  for (int j = 0; j < IPT; ++j) {
    const int c0 = (threadIdx.x + j * kRowT) * 16;
    if (tap && tap_normed && live) {
#pragma unroll
      for (int e = 0; e < 16; ++e)
        if (c0 + e < hidden) tap[(size_t)t * hidden + c0 + e] = (x[j][e] * r) * gv[j][e];
    }
#pragma unroll
    for (int e = 0; e < 16; ++e) x[j][e] *= gv[j][e];
  }
  quantize_row<kRowT, IPT>(x, t, ks, r, codes, scale, redq);
}

// Pairs of q and k (j, j + d / 2) by rotation; then v transposed, the token
// fastest, so that a wave's stores fall into runs of cache slots.
__global__ __launch_bounds__(256) void k_rope_store(RopeStoreArgs a) {
  const int d = a.head_dim, half = d / 2;
  const int qd = a.n_heads * d, kvd = a.n_kv * d, width = qd + 2 * kvd;
  const int pairs = a.n_tok * (a.n_heads + a.n_kv) * half;
  const int i = blockIdx.x * 256 + threadIdx.x;
  if (i < pairs) {
    const int t = i / ((a.n_heads + a.n_kv) * half), p = i - t * (a.n_heads + a.n_kv) * half;
    const int head = p / half, j = p - head * half;
    const float *y = a.y + (size_t)t * width + head * d + j;
    const float2 cs = a.rope[t * half + j];
    const float x1 = y[0], x2 = y[half];
    uint16_t *dst = head < a.n_heads
                        ? a.q + ((size_t)t * a.n_heads + head) * d
                        : a.kc + ((size_t)(head - a.n_heads) * a.cap + a.kv_len + t) * d;
    dst[j] = f2bf(x1 * cs.x - x2 * cs.y);
    dst[j + half] = f2bf(x2 * cs.x + x1 * cs.y);
  } else if (i - pairs < a.n_tok * kvd) {
    const int v = i - pairs, e = v / a.n_tok, t = v - e * a.n_tok;
    a.vc[(size_t)e * a.cap + a.kv_len + t] = f2bf(a.y[(size_t)t * width + qd + kvd + e]);
  }
}

template <int IPT>
__global__ __launch_bounds__(kRowT) void k_swiglu_quant(const float *__restrict__ y, int n_tok,
                                                        int ffn, int ks, int vec, uint8_t *codes,
                                                        float *scale) {
  __shared__ uint32_t red[kRowT / 64];
  const int t = blockIdx.x;
  const float *gate = y + (size_t)t * 2 * ffn, *up = gate + ffn;
  float x[IPT][16], u[IPT][16];
#pragma unroll
  for (int j = 0; j < IPT; ++j)
#pragma unroll
    for (int q = 0; q < 4; ++q) {
      const int c = (threadIdx.x + j * kRowT) * 16 + 4 * q;
      f32x4 a = {0.f, 0.f, 0.f, 0.f}, b = a;
      if (t < n_tok && c < ffn) {
        if (vec) {
          a = *(const f32x4 *)(gate + c);
          b = *(const f32x4 *)(up + c);
        } else {
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            a[e] = c + e < ffn ? gate[c + e] : 0.0f;
            b[e] = c + e < ffn ? up[c + e] : 0.0f;
          }
        }
      }
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        x[j][4 * q + e] = a[e];
        u[j][4 * q + e] = b[e];
      }
    }
#pragma unroll
  for (int j = 0; j < IPT; ++j)
#pragma unroll
    for (int e = 0; e < 16; ++e) {
      // silu(g) = g / (1 + e^-g) with the hardware exp2 and reciprocal: their
      // few units of 2^-24 are far below a code's step
      const float g = x[j][e];
      x[j][e] = g * __builtin_amdgcn_rcpf(1.0f + __builtin_amdgcn_exp2f(g * -1.44269504f)) * u[j][e];
    }
  quantize_row<kRowT, IPT>(x, t, ks, 1.0f, codes, scale, red);
}

}  // namespace

hipError_t launch_norm_quant(float *h, const float *delta, const float *g, int hidden, int n_tok,
                             float eps, uint8_t *codes, float *scale, hipStream_t s, float *tap,
                             int tap_normed) {
  const int ks = linear_geom(1, hidden).ks, ipt = ceil_div(ks * 4, kRowT);
  const dim3 grid(round_up(n_tok, 16)), block(kRowT);
  if (hidden % 8 != 0) return hipErrorInvalidValue;
  if (ipt == 1)
    hipLaunchKernelGGL(k_norm_quant<1>, grid, block, 0, s, h, delta, g, hidden, ks, n_tok, eps, codes,
                       scale, tap, tap_normed);
  else if (ipt == 2)
    hipLaunchKernelGGL(k_norm_quant<2>, grid, block, 0, s, h, delta, g, hidden, ks, n_tok, eps, codes,
                       scale, tap, tap_normed);
  else
    return hipErrorInvalidValue;
  return hipGetLastError();
}

hipError_t launch_rope_store(const RopeStoreArgs &a, hipStream_t s) {
  const int items = a.n_tok * ((a.n_heads + a.n_kv) * (a.head_dim / 2) + a.n_kv * a.head_dim);
  hipLaunchKernelGGL(k_rope_store, dim3(ceil_div(items, 256)), dim3(256), 0, s, a);
  return hipGetLastError();
}

hipError_t launch_swiglu_quant(const float *y, int n_tok, int ffn, uint8_t *codes, float *scale,
                               hipStream_t s) {
  const int ks = linear_geom(1, ffn).ks, ipt = ceil_div(ks * 4, kRowT);
  const dim3 grid(round_up(n_tok, 16)), block(kRowT);
  const int vec = ffn % 4 == 0;
  switch (ipt) {
#define SB_IPT(i)                                                                               \
  case i:                                                                                       \
    hipLaunchKernelGGL(k_swiglu_quant<i>, grid, block, 0, s, y, n_tok, ffn, ks, vec, codes, scale); \
    break;
    SB_IPT(1) SB_IPT(2) SB_IPT(3) SB_IPT(4)
#undef SB_IPT
    default: return hipErrorInvalidValue;
  }
  return hipGetLastError();
}

}  // namespace sb
