// Projections in 8-bit integers: y[t][r] = sx[t] sw[r] sum_k x[t][k] w[r][k],
// codes in [-127, 127] with a scale per token and per output channel, sums in
// 32-bit integers (exact for up to 2^17 inputs).
//
// What bounds it: the weights' bytes, m k, read once, up to some 100 rows; then the
// activations' way to the compute units, as every workgroup reads all n k of them
// from the L2.  Weights and activations lie in the operand order of the 16x16x64
// integer matrix instruction, 16 bytes per lane and k-step of 64, tiles of 16
// channels or tokens.  Two kernels (linear_plan has the rule and both sides'
// times):
// - k_linear, few rows: both operands straight to registers; a workgroup owns NT
//   weight tiles and TT token tiles, its waves split K, so every wave streams its
//   own stretch of the tiles with nothing shared until the end, where the waves'
//   sums meet in LDS.  22016 x 4096, 33 rows: 19 us, 4.8 TB/s.
// - k_linear_ring, many rows: 128 or 256 channels and all rows per workgroup, so
//   that activations are read once per that many channels, through a ring of LDS
//   stages that its waves share; the weights, each wave's own, straight to
//   registers.  57344 x 8192, 129 rows: 91 us, 5.2 TB/s (k_linear: 171).
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

// Outputs r .. r + 3 (r a multiple of 4) of token t from their sums.
__device__ __forceinline__ void store_scaled(const LinearArgs &a, int t, int r, i32x4 v, f32x4 sw) {
  const float sx = a.x_scale[t];
  f32x4 y;
#pragma unroll
  for (int e = 0; e < 4; ++e) y[e] = (float)v[e] * (sx * sw[e]);
  float *dst = a.y + (size_t)t * a.m + r;
  if (a.vec && r < a.m) {
    *(f32x4 *)dst = y;
  } else {
#pragma unroll
    for (int e = 0; e < 4; ++e)
      if (r + e < a.m) dst[e] = y[e];
  }
}

// NT weight tiles x TT token tiles, NW waves; kU k-steps are in flight while
// the kU before them are multiplied (four where registers allow: level on long K,
// 0.3 to 1.5 us slower on K of 768 to 5120).
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
      // past the wave's stretch: an offset past both buffers (4 MB at most), which reads zeros
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
      store_scaled(a, t, r, v, *(const f32x4 *)(a.w_scale + r));
    }
  }
}

// More token tiles: a wave owns NT weight tiles and all TT token tiles, the
// kRingWaves waves of a workgroup kRingWaves NT weight tiles.  The activations of a
// stage, KS k-steps, are read once per workgroup, by direct-to-LDS loads into a ring
// of three stages (two in flight while one is multiplied), the weights beside them
// into as many sets of registers.  Their non-temporal hint is worth 118 -> 100 us
// (57344 x 8192, 129 rows, weights from HBM); weights through the ring as well, which
// then holds half as many k-steps, measured 118 too.  grid: tile groups x K ranges;
// K range `split` of several leaves its sums, 32-bit integers, in
// part[split][n_tok][16 tiles].
constexpr int kRingWaves = 8, kRingMaxSplits = 8;
typedef __attribute__((address_space(3))) void lds_void;

template <int NT, int TT, int KS>
__global__ __launch_bounds__(64 * kRingWaves) void k_linear_ring(LinearArgs a) {
  constexpr int WT = kRingWaves * NT;  // weight tiles of a workgroup
  constexpr int F = TT * KS;           // activation fragments of a stage
  constexpr int LPW = (F + kRingWaves - 1) / kRingWaves;  // of them per wave
  // the waves without a fragment in the last turn load zeros into one more
  constexpr int kBytes = (F + (F % kRingWaves != 0)) * 1024;
  __shared__ __attribute__((aligned(16))) char r0[kBytes], r1[kBytes], r2[kBytes];
  const int w = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lane = threadIdx.x & 63;
  const int split = blockIdx.x % a.splits, tile0 = blockIdx.x / a.splits * WT;
  const int tile_bytes = a.ks * 1024;
  const int wt0 = tile0 + w * NT;  // the wave's own tiles; those past the last read zeros
  const int wn = min(NT, a.tiles - wt0);
  const __amdgpu_buffer_rsrc_t wrs =
      uniform_rsrc(a.w + (size_t)min(wt0, a.tiles - 1) * tile_bytes, max(wn, 0) * tile_bytes);
  const __amdgpu_buffer_rsrc_t xrs = uniform_rsrc(a.x, a.ttiles * tile_bytes);
  const int s0 = (int)((int64_t)a.ks * split / a.splits), s1 = (int)((int64_t)a.ks * (split + 1) / a.splits);
  constexpr int kPast = 0x7fff0000;  // past both buffers: reads zeros
  struct Weights {
    i32x4 f[KS][NT];
  };
  // Stage at k-step s: activation fragment f, k-step f / TT of token tile f % TT, to
  // LDS, and the wave's own weights.  Steps past s1 and tiles past the last read
  // zeros (offsets: at most 16 tiles of 512 KB).
  auto issue = [&](int s, char *dst, Weights &b) {
#pragma unroll
    for (int j = 0; j < LPW; ++j) {
      const int f = w + j * kRingWaves;  // uniform
      const int k = s + f / TT, t = f % TT;
      const bool in = f < F && k < s1 && t < a.ttiles;
      __builtin_amdgcn_raw_ptr_buffer_load_lds(xrs, (lds_void *)(dst + min(f, F) * 1024), 16,
                                               in ? (t * a.ks + k) * 1024 + lane * 16 : kPast, 0, 0, 0);
    }
#pragma unroll
    for (int k = 0; k < KS; ++k)
#pragma unroll
      for (int i = 0; i < NT; ++i)
        b.f[k][i] = __builtin_amdgcn_raw_buffer_load_b128(
            wrs, s + k < s1 && i < wn ? (i * a.ks + s + k) * 1024 + lane * 16 : kPast, 0, kNonTemporal);
  };
  i32x4 acc[NT][TT];
#pragma unroll
  for (int i = 0; i < NT; ++i)
#pragma unroll
    for (int j = 0; j < TT; ++j) acc[i][j] = i32x4{0, 0, 0, 0};
  Weights b0, b1, b2;
  issue(s0, r0, b0);
  issue(s0 + KS, r1, b1);
  // The stage at s is there once every wave has waited for its own loads of it
  // (one later stage may be in flight) and met the others; then the buffer of the
  // stage before is free.
  auto round = [&](int s, const char *cur, const Weights &b, char *nxt, Weights &nb) {
    asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)\n\ts_barrier" ::"n"(LPW + KS * NT) : "memory");
    issue(s + 2 * KS, nxt, nb);
    __builtin_amdgcn_sched_barrier(0);
    if (s >= s1) return;
    const char *frag = cur + lane * 16;
#pragma unroll
    for (int k = 0; k < KS; ++k)
#pragma unroll
      for (int j = 0; j < TT; ++j) {
        const i32x4 xf = *(const i32x4 *)(frag + (k * TT + j) * 1024);
#pragma unroll
        for (int i = 0; i < NT; ++i) acc[i][j] = mfma16i(b.f[k][i], xf, acc[i][j]);
      }
  };
  for (int s = s0; s < s1; s += 3 * KS) {
    round(s, r0, b0, r2, b2);
    round(s + KS, r1, b1, r0, b0);
    round(s + 2 * KS, r2, b2, r1, b1);
  }
  asm volatile("s_waitcnt vmcnt(0)" ::: "memory");  // loads into LDS still in flight
  // element e of lane l is channel 4 (l / 16) + e of the tile, token l % 16
#pragma unroll
  for (int i = 0; i < NT; ++i) {
    const int r = (tile0 + w * NT + i) * 16 + 4 * (lane >> 4);
    if (r >= a.tiles * 16) continue;
    const f32x4 sw = *(const f32x4 *)(a.w_scale + r);
#pragma unroll
    for (int j = 0; j < TT; ++j) {
      const int t = j * 16 + (lane & 15);
      if (t >= a.n_tok) continue;
      if (a.splits > 1) {
        *(i32x4 *)(a.part + ((size_t)split * a.n_tok + t) * a.tiles * 16 + r) = acc[i][j];
        continue;
      }
      store_scaled(a, t, r, acc[i][j], sw);
    }
  }
}

// The sums of the K ranges, scaled: four channels a thread.
__global__ __launch_bounds__(256) void k_linear_join(LinearArgs a) {
  const int quads = a.tiles * 4, i = blockIdx.x * 256 + threadIdx.x;
  const int t = i / quads, r = (i - t * quads) * 4;
  if (t >= a.n_tok) return;
  const size_t stride = (size_t)a.n_tok * a.tiles * 16;
  const int32_t *p = a.part + (size_t)t * a.tiles * 16 + r;
  i32x4 v = *(const i32x4 *)p;
  for (int k = 1; k < a.splits; ++k) v += *(const i32x4 *)(p + k * stride);
  store_scaled(a, t, r, v, *(const f32x4 *)(a.w_scale + r));
}

template <int NT, int TT, int NW>
hipError_t launch_form(const LinearArgs &a, hipStream_t s) {
  const int groups = ceil_div(a.tiles, NT);
  hipLaunchKernelGGL((k_linear<NT, TT, NW>), dim3(groups * a.tblocks), dim3(64 * NW), 0, s, a);
  return hipGetLastError();
}

// Most weight tiles of a workgroup of k_linear: what the accumulators leave
// registers for.
constexpr int most_tiles(int tt) { return tt <= 2 ? 8 : tt == 3 ? 6 : tt == 4 ? 5 : 4; }

template <int TT>
hipError_t launch_tt(const LinearArgs &a, int nt, hipStream_t s) {
  constexpr int NW = TT <= 4 ? 8 : 4, M = most_tiles(TT);
  switch (nt) {
    case 1: return launch_form<1, TT, NW>(a, s);
    case 2: return launch_form<2, TT, NW>(a, s);
    case 3: return launch_form<3, TT, NW>(a, s);
    case 4: return launch_form<4, TT, NW>(a, s);
    case 5: return launch_form<M < 5 ? 4 : 5, TT, NW>(a, s);
    case 6: return launch_form<M < 6 ? 4 : 6, TT, NW>(a, s);
    case 8: return launch_form<M < 8 ? 4 : 8, TT, NW>(a, s);
    default: return hipErrorInvalidValue;
  }
}

template <int NT, int TT>
hipError_t launch_ring(const LinearArgs &a, hipStream_t s) {
  // Twice as long stages: 57344 x 8192, 65 rows 84.5 -> 91.7 us, 129 rows 98 -> 103,
  // 5120 x 13824, 33 rows 24.6 -> 27.2.  (Two weight tiles and twelve or more token
  // tiles: 1 for 2, 256 rows 140 -> 150.)
  constexpr int KS = TT <= 3 ? 4 : TT <= 9 || NT == 2 ? 2 : 1;
  const int groups = ceil_div(a.tiles, kRingWaves * NT);
  hipLaunchKernelGGL((k_linear_ring<NT, TT, KS>), dim3(groups * a.splits), dim3(64 * kRingWaves), 0,
                     s, a);
  if (a.splits > 1)
    hipLaunchKernelGGL(k_linear_join, dim3(ceil_div(a.n_tok * a.tiles * 4, 256)), dim3(256), 0, s, a);
  return hipGetLastError();
}

// Token tiles up to the next form: the multiplications of a tile that is not
// there cost nothing next to the weights' bytes.
template <int NT>
hipError_t launch_ring_tt(const LinearArgs &a, hipStream_t s) {
  if (a.ttiles <= 2) return launch_ring<NT, 2>(a, s);
  if (a.ttiles <= 3) return launch_ring<NT, 3>(a, s);
  if (a.ttiles <= 5) return launch_ring<NT, 5>(a, s);
  if (a.ttiles <= 7) return launch_ring<NT, 7>(a, s);
  if (a.ttiles <= 9) return launch_ring<NT, 9>(a, s);
  if (a.ttiles <= 12) return launch_ring<NT, 12>(a, s);
  return launch_ring<NT, 16>(a, s);
}

}  // namespace

// The kernel and its tiles by what a compute unit has to bring in, in KB (1 KB per
// tile and k-step), as its fill rate bounds both kernels; a round of workgroups
// costs 100 KB more.  For k_linear that is rounds (nt + tt) ks, which is least
// where the tiles make one even round; measured, by nt, us:
//   12288 x 4096, 33 rows    2: 18.9   3: 15.0   4: 16.3   6: 19.6
//   22016 x 4096, 33 rows    3: 24.3   4: 27.3   5: 31.0   6: 22.5
//   57344 x 8192, 33 rows    2: 103    4: 94.8   5: 90.8   6: 99.8
// The ring's bytes count 1.3 times (1.25 with two tiles a wave: stages and
// barriers), K ranges 300 KB (the join's launch) and twice their sums.  (45000 x
// 5120 with one tile a wave, or k_linear, against two: 49 rows 58.7 / 48.2, 65 rows
// 63.2 / 50.2.)  Measured, k_linear / the ring with one / with two tiles a wave, with the
// rows' quantisation, us:
//   rows                    17                  33                  65                  129
//   4096 x 4096      9.3 / 13.7 / 15.5  10.4 / 15.7 / 17.4  12.3 / 18.3 / 20.2  14.0 / 23.4 / 26.8
//   12288 x 4096    14.5 / 18.0 / 21.7  15.4 / 19.5 / 24.0  18.0 / 22.7 / 25.5  26.5 / 28.7 / 31.3
//   22016 x 4096    21.2 / 25.1 / 31.4  22.5 / 26.2 / 33.0  28.0 / 28.3 / 34.2  43.7 / 33.6 / 41.5
//   5120 x 13824    26.6 / 22.7 / 26.8  30.1 / 24.6 / 29.3  36.5 / 28.3 / 34.0  43.3 / 34.8 / 39.2
//   8192 x 28672    53.7 / 50.8 / 53.0  59.2 / 52.8 / 54.5  74.8 / 60.6 / 60.4   101 / 74.2 / 75.1
//   57344 x 8192    85.4 / 86.4 / 86.2  89.5 / 88.1 / 87.9   114 / 94.9 / 85.4   177 / 116  / 95.6
// One token tile is always k_linear's.
LinearPlan linear_plan(int tiles, int ks, int n_tok) {
  LinearPlan p{};
  const int ttiles = ceil_div(n_tok, 16);
  p.splits = 1;
  p.tblocks = ceil_div(ttiles, kLinearMaxTokenTiles);
  const int tt = ceil_div(ttiles, p.tblocks);
  int64_t best = INT64_MAX;
  for (const int nt : {8, 6, 5, 4, 3, 2, 1}) {
    if (nt > most_tiles(tt)) continue;
    const int64_t rounds = ceil_div(ceil_div(tiles, nt) * p.tblocks, kAttnCUs);
    const int64_t cost = rounds * ((int64_t)(nt + tt) * ks + 100);
    if (cost < best) {
      best = cost;
      p.nt = nt;
    }
  }
  for (int r = 1; r <= 2 && ttiles >= 2; ++r) {
    const int groups = ceil_div(tiles, kRingWaves * r);
    // K ranges of eight k-steps or more, up to a workgroup for every compute unit
    int splits = kAttnCUs / groups;
    if (splits > kRingMaxSplits) splits = kRingMaxSplits;
    if (splits > ks / 8) splits = ks / 8;
    if (splits < 1) splits = 1;
    const int64_t rounds = ceil_div(groups * splits, kAttnCUs);
    const int64_t kb = (int64_t)(kRingWaves * r + ttiles) * ceil_div(ks, splits) * (r == 2 ? 125 : 130) / 100;
    const int64_t sums = splits > 1 ? 300 + (int64_t)splits * ttiles * tiles / 64 : 0;
    if (rounds * (kb + 100) + sums < best) {
      best = rounds * (kb + 100) + sums;
      p.ring_tiles = r;
      p.splits = splits;
    }
  }
  return p;
}

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

size_t linear_part_bytes(int m, int k, int max_rows) {
  const LinearGeom g = linear_geom(m, k);
  size_t most = 0;
  for (int rows = max_rows; rows > 0; rows = round_up(rows, 16) - 16) {  // the most of each plan
    const int splits = linear_plan(g.tiles, g.ks, rows).splits;
    const size_t b = splits > 1 ? (size_t)splits * rows * g.tiles * 16 * sizeof(int32_t) : 0;
    if (b > most) most = b;
  }
  return most;
}

hipError_t launch_linear(const LinearArgs &args, hipStream_t s) {
  LinearArgs a = args;
  a.vec = a.m % 4 == 0 && ((uintptr_t)a.y & 15) == 0;
  a.ttiles = ceil_div(a.n_tok, 16);
  const LinearPlan p = linear_plan(a.tiles, a.ks, a.n_tok);
  a.tblocks = p.tblocks;
  a.splits = p.splits;
  if (p.ring_tiles == 1) return launch_ring_tt<1>(a, s);
  if (p.ring_tiles == 2) return launch_ring_tt<2>(a, s);
  switch (ceil_div(a.ttiles, a.tblocks)) {
    case 1: return launch_tt<1>(a, p.nt, s);
    case 2: return launch_tt<2>(a, p.nt, s);
    case 3: return launch_tt<3>(a, p.nt, s);
    case 4: return launch_tt<4>(a, p.nt, s);
    case 5: return launch_tt<5>(a, p.nt, s);
    case 6: return launch_tt<6>(a, p.nt, s);
    case 7: return launch_tt<7>(a, p.nt, s);
    case 8: return launch_tt<8>(a, p.nt, s);
    default: return hipErrorInvalidValue;
  }
}

}  // namespace sb
