// Projections in 8-bit integers: y[t][r] = sx[t] sw[r] sum_k x[t][k] w[r][k],
// codes in [-127, 127] with a scale per token and per output channel, sums in
// 32-bit integers (exact for up to 2^17 inputs).
//
// The product streams every weight tile (16 channels) from HBM once, 16 bytes
// per lane and k-step of 64 in the operand order of the 16x16x64 integer
// matrix instruction, straight into registers; the activations (all rows: at
// most 256 x 28672 bytes) come the same way out of the L2.  A workgroup owns NT
// weight tiles and TT token tiles; its waves split K, so every wave streams its
// own stretch of the tiles with nothing shared until the end, where the waves'
// sums meet in LDS.
#include <math.h>

#include "sb_internal_fwd.h"
#include "sb_quant_device.h"

namespace sb {
namespace {

// ---- weights ---------------------------------------------------------------

// One workgroup per tile: 16 threads per output channel find its largest
// magnitude, then write its codes (the second read comes out of the L2).
// Channels past the last and columns past k are zeros.
__global__ __launch_bounds__(256) void k_linear_pack(LinearPackArgs a) {
  const int r = threadIdx.x & 15, part = threadIdx.x >> 4;
  const int row = blockIdx.x * 16 + r;
  const bool there = row < a.rows[0] + a.rows[1] + a.rows[2];
  int at = row;
  const uint16_t *src = a.src[0];
  if (at >= a.rows[0]) {
    at -= a.rows[0];
    src = a.src[1];
    if (at >= a.rows[1]) {
      at -= a.rows[1];
      src = a.src[2];
    }
  }
  src += there ? (size_t)at * a.k : 0;
  const bool vec = a.k % 8 == 0 && ((uintptr_t)src & 15) == 0;
  auto load = [&](int item, uint32_t (&w)[8]) {  // 16 columns, two per word
    const int c0 = item * 16;
    if (vec) {
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        const uint4 x = there && c0 + 8 * h < a.k ? *(const uint4 *)(src + c0 + 8 * h)
                                                  : make_uint4(0, 0, 0, 0);
        w[4 * h] = x.x;
        w[4 * h + 1] = x.y;
        w[4 * h + 2] = x.z;
        w[4 * h + 3] = x.w;
      }
    } else {
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        const int c = c0 + 2 * e;
        w[e] = (there && c < a.k ? src[c] : 0u) | (there && c + 1 < a.k ? (uint32_t)src[c + 1] << 16 : 0u);
      }
    }
  };
  __shared__ uint32_t red[16][17];
  uint32_t top = 0;
  for (int item = part; item < a.ks * 4; item += 16) {
    uint32_t w[8];
    load(item, w);
#pragma unroll
    for (int e = 0; e < 8; ++e) top = max(top, max(w[e] & 0x7fffu, (w[e] >> 16) & 0x7fffu));
  }
  red[part][r] = top;
  __syncthreads();
  top = 0;
#pragma unroll
  for (int i = 0; i < 16; ++i) top = max(top, red[i][r]);
  const bool finite = top < 0x7f80u;
  const float amax = __uint_as_float(top << 16);
  if (part == 0) a.scale[row] = finite ? amax / 127.0f : NAN;
  for (int item = part; item < a.ks * 4; item += 16) {
    uint32_t w[8];
    load(item, w);
    float x[16];
#pragma unroll
    for (int e = 0; e < 16; ++e) x[e] = bf2f((uint16_t)(w[e >> 1] >> (16 * (e & 1))));
    *(uint4 *)(a.codes + item_offset(row, item, a.ks)) = codes16(x, amax, finite && top != 0);
  }
}

// ---- activations -----------------------------------------------------------

constexpr int kRowT = 512;

// One workgroup per row, the row in registers (one read); rows past n_tok are
// zeros, so that the product's last token tile is whole.
template <typename T, int IPT>
__global__ __launch_bounds__(kRowT) void k_quant_rows(const T *__restrict__ x, int n_tok, int k,
                                                      int ks, int vec, uint8_t *codes,
                                                      float *scale) {
  __shared__ uint32_t red[kRowT / 64];
  const int row = blockIdx.x;
  const T *src = x + (size_t)row * k;
  float v[IPT][16];
#pragma unroll
  for (int j = 0; j < IPT; ++j) {
    const int c0 = (threadIdx.x + j * kRowT) * 16;
    const bool in = row < n_tok && c0 < k;
    if (sizeof(T) == 2 && vec) {
      uint4 w[2];
#pragma unroll
      for (int h = 0; h < 2; ++h)
        w[h] = in && c0 + 8 * h < k ? *(const uint4 *)(src + c0 + 8 * h) : make_uint4(0, 0, 0, 0);
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        const uint32_t d[4] = {w[h].x, w[h].y, w[h].z, w[h].w};
#pragma unroll
        for (int e = 0; e < 8; ++e) v[j][8 * h + e] = bf2f((uint16_t)(d[e >> 1] >> (16 * (e & 1))));
      }
    } else if (sizeof(T) == 4 && vec) {
#pragma unroll
      for (int q = 0; q < 4; ++q) {
        const f32x4 w = in && c0 + 4 * q < k ? *(const f32x4 *)(src + c0 + 4 * q) : f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int e = 0; e < 4; ++e) v[j][4 * q + e] = w[e];
      }
    } else {
#pragma unroll
      for (int e = 0; e < 16; ++e) {
        if (in && c0 + e < k) {
          if (sizeof(T) == 2)
            v[j][e] = bf2f((uint16_t)src[c0 + e]);
          else
            v[j][e] = (float)src[c0 + e];
        } else {
          v[j][e] = 0.0f;
        }
      }
    }
  }
  quantize_row<kRowT, IPT>(v, row, ks, 1.0f, codes, scale, red);
}

// ---- the product -------------------------------------------------------------

__device__ __forceinline__ i32x4 mfma16i(i32x4 a, i32x4 b, i32x4 c) {
  return __builtin_amdgcn_mfma_i32_16x16x64_i8(a, b, c, 0, 0, 0);
}

// NT weight tiles x TT token tiles, NW waves; kU k-steps are in flight while
// the kU before them are multiplied.
constexpr int kU = 2;
template <int NT, int TT, int NW>
__global__ __launch_bounds__(64 * NW) void k_linear(LinearArgs a) {
  constexpr int P = NT * TT;               // pairs of a weight and a token tile
  constexpr int PR = 64 / NW < P ? 64 / NW : P;  // pairs summed over the waves per round (64 KB)
  __shared__ i32x4 red[NW][PR][64];
  const int w = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lane = threadIdx.x & 63;
  // Work unit (tile group, token block), XCD-major, the token block fastest (the
  // workgroups of one tile group share its weights through the L2).
  const int xcd = blockIdx.x & 7, left = gridDim.x & 7;
  const int unit = xcd * (gridDim.x >> 3) + (xcd < left ? xcd : left) + (blockIdx.x >> 3);
  const int tile0 = unit / a.tblocks * NT, tt0 = unit % a.tblocks * TT;
  const int tile_bytes = a.ks * 1024;
  const int wn = min(NT, a.tiles - tile0), xn = min(TT, a.ttiles - tt0);
  // tiles past the last repeat it: their sums are not stored
  const __amdgpu_buffer_rsrc_t wrs = uniform_rsrc(a.w + (size_t)tile0 * tile_bytes, wn * tile_bytes);
  const __amdgpu_buffer_rsrc_t xrs = uniform_rsrc(a.x + (size_t)tt0 * tile_bytes, xn * tile_bytes);
  const int s0 = a.ks * w / NW, s1 = a.ks * (w + 1) / NW;
  struct Buf {
    i32x4 w[kU][NT], x[kU][TT];
  };
  auto load = [&](Buf &b, int s) {
#pragma unroll
    for (int u = 0; u < kU; ++u) {
      // past the wave's stretch: an offset past both buffers (2 MB and 4 MB at
      // most), which reads zeros
      const int vo = s + u < s1 ? (s + u) * 1024 + lane * 16 : 0x7fff0000;
#pragma unroll
      for (int i = 0; i < NT; ++i)
        b.w[u][i] = __builtin_amdgcn_raw_buffer_load_b128(wrs, vo, min(i, wn - 1) * tile_bytes, kNonTemporal);
#pragma unroll
      for (int j = 0; j < TT; ++j)
        b.x[u][j] = __builtin_amdgcn_raw_buffer_load_b128(xrs, vo, min(j, xn - 1) * tile_bytes, 0);
    }
  };
  i32x4 acc[NT][TT];
#pragma unroll
  for (int i = 0; i < NT; ++i)
#pragma unroll
    for (int j = 0; j < TT; ++j) acc[i][j] = i32x4{0, 0, 0, 0};
  auto multiply = [&](const Buf &b) {
#pragma unroll
    for (int u = 0; u < kU; ++u)
#pragma unroll
      for (int i = 0; i < NT; ++i)
#pragma unroll
        for (int j = 0; j < TT; ++j) acc[i][j] = mfma16i(b.w[u][i], b.x[u][j], acc[i][j]);
  };
  Buf b0, b1;
  load(b0, s0);
  for (int s = s0; s < s1; s += 2 * kU) {
    load(b1, s + kU);
    __builtin_amdgcn_sched_barrier(0);
    multiply(b0);
    load(b0, s + 2 * kU);
    __builtin_amdgcn_sched_barrier(0);
    multiply(b1);
  }
  // ---- the waves' sums, PR pairs at a time; element e of lane l is channel
  // 4 (l / 16) + e of the tile, token l % 16
#pragma unroll
  for (int p0 = 0; p0 < P; p0 += PR) {
    if (p0) __syncthreads();
#pragma unroll
    for (int p = 0; p < PR; ++p)
      if (p0 + p < P) red[w][p][lane] = acc[(p0 + p) / TT][(p0 + p) % TT];
    __syncthreads();
    for (int i = threadIdx.x; i < PR * 64; i += 64 * NW) {
      const int p = p0 + (i >> 6), ln = i & 63;
      if (p >= P) continue;
      i32x4 v = red[0][i >> 6][ln];
#pragma unroll
      for (int k = 1; k < NW; ++k) v += red[k][i >> 6][ln];
      const int r = (tile0 + p / TT) * 16 + 4 * (ln >> 4), t = (tt0 + p % TT) * 16 + (ln & 15);
      if (t >= a.n_tok || r >= a.m) continue;
      const f32x4 sw = *(const f32x4 *)(a.w_scale + r);
      const float sx = a.x_scale[t];
      f32x4 y;
#pragma unroll
      for (int e = 0; e < 4; ++e) y[e] = (float)v[e] * (sx * sw[e]);
      float *dst = a.y + (size_t)t * a.m + r;
      if (a.vec) {
        *(f32x4 *)dst = y;
      } else {
#pragma unroll
        for (int e = 0; e < 4; ++e)
          if (r + e < a.m) dst[e] = y[e];
      }
    }
  }
}

template <int NT, int TT, int NW>
hipError_t launch_form(const LinearArgs &a, hipStream_t s) {
  const int groups = ceil_div(a.tiles, NT);
  hipLaunchKernelGGL((k_linear<NT, TT, NW>), dim3(groups * a.tblocks), dim3(64 * NW), 0, s, a);
  return hipGetLastError();
}

template <int TT>
hipError_t launch_tt(const LinearArgs &a, int nt, hipStream_t s) {
  switch (nt) {
    case 1: return launch_form<1, TT, 8>(a, s);
    case 2: return launch_form<2, TT, TT <= 4 ? 8 : 4>(a, s);
    case 4: return launch_form<4, TT, TT <= 4 ? 8 : 4>(a, s);
    default: return hipErrorInvalidValue;
  }
}

}  // namespace

LinearGeom linear_geom(int m, int k) {
  LinearGeom g{};
  g.tiles = ceil_div(m, 16);
  g.ks = round_up(ceil_div(k, 64), 4);
  g.scales = (size_t)g.tiles * g.ks * 1024;
  g.bytes = g.scales + (size_t)g.tiles * 16 * sizeof(float);
  return g;
}

hipError_t launch_linear_pack(const LinearPackArgs &args, hipStream_t s) {
  LinearPackArgs a = args;
  const LinearGeom g = linear_geom(a.rows[0] + a.rows[1] + a.rows[2], a.k);
  a.ks = g.ks;
  a.scale = (float *)(a.codes + g.scales);
  hipLaunchKernelGGL(k_linear_pack, dim3(g.tiles), dim3(256), 0, s, a);
  return hipGetLastError();
}

hipError_t launch_quant_rows(const void *x, bool bf16, int n_tok, int k, uint8_t *codes,
                             float *scale, hipStream_t s) {
  const int ks = linear_geom(1, k).ks, ipt = ceil_div(ks * 4, kRowT);
  const dim3 grid(round_up(n_tok, 16)), block(kRowT);
  // 16-byte loads where every row starts on one
  const int vec = k % (bf16 ? 8 : 4) == 0 && ((uintptr_t)x & 15) == 0;
#define SB_IPT(i)                                                                                \
  case i:                                                                                        \
    if (bf16)                                                                                    \
      hipLaunchKernelGGL((k_quant_rows<uint16_t, i>), grid, block, 0, s, (const uint16_t *)x,    \
                         n_tok, k, ks, vec, codes, scale);                                       \
    else                                                                                         \
      hipLaunchKernelGGL((k_quant_rows<float, i>), grid, block, 0, s, (const float *)x, n_tok, k,\
                         ks, vec, codes, scale);                                                 \
    break;
  switch (ipt) {
    SB_IPT(1) SB_IPT(2) SB_IPT(3) SB_IPT(4)
    default: return hipErrorInvalidValue;
  }
#undef SB_IPT
  return hipGetLastError();
}

// Tiles per workgroup: as many (up to four) as leave a workgroup for every
// compute unit.
hipError_t launch_linear(const LinearArgs &args, hipStream_t s) {
  LinearArgs a = args;
  a.vec = a.m % 4 == 0 && ((uintptr_t)a.y & 15) == 0;
  a.ttiles = ceil_div(a.n_tok, 16);
  a.tblocks = ceil_div(a.ttiles, kLinearMaxTokenTiles);
  const int tt = ceil_div(a.ttiles, a.tblocks);
  int nt = 4;
  while (nt > 1 && ceil_div(a.tiles, nt) * a.tblocks < kAttnCUs) nt /= 2;
  switch (tt) {
    case 1: return launch_tt<1>(a, nt, s);
    case 2: return launch_tt<2>(a, nt, s);
    case 3: return launch_tt<3>(a, nt, s);
    case 4: return launch_tt<4>(a, nt, s);
    case 5: return launch_tt<5>(a, nt, s);
    case 6: return launch_tt<6>(a, nt, s);
    case 7: return launch_tt<7>(a, nt, s);
    case 8: return launch_tt<8>(a, nt, s);
    default: return hipErrorInvalidValue;
  }
}

}  // namespace sb
