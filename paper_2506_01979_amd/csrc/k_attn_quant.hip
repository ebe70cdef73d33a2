// Branch-masked attention over a prefix cache held in 8 bits, with a 16-bit
// tail behind it (the committed tokens that fill no block yet, then the
// tree's rows): the attention of k_attn.hip, one softmax over both parts.
//
// Flash-decoding split as there: the blocks of every KV head are cut into c8
// ranges and the tail into ct, one workgroup each (and per block of at most 48
// query rows), and the merge kernels of k_attn.hip combine the ranges.  Every
// wave streams key blocks of its own (of the range, every fourth) with a
// running softmax for all of the workgroup's rows, so that nothing is shared
// between the waves until the end: no barrier in the loop, every code is
// converted once per workgroup, and the four waves' sums meet in LDS after the
// last block.
//
// An 8-bit block (64 keys): its codes come in operand order, 16 bytes per lane
// and fragment, straight into registers, and are widened to binary16 there,
// where both formats are exact: int8 by placing the byte under the exponent of
// 1024 and subtracting 1152, e4m3 by the conversion instruction.  The scales
// never touch the codes: K's multiplies the scores with the softmax factor, V's
// multiplies the softmax weights,
//   S^T = K Q^T;  w = exp2(s kscale c - m + log2 r);  l += w / r;  O^T += V^T w^T,
//   r = vscale 2^15 / (the largest vscale of the wave's blocks),
// so that w <= 2^15 is binary16 to 11 bits down to 2^-29 of the largest
// weight.  Those 11 bits are the products' rounding point: an eighth of what
// the output's bfloat16 keeps, and one matrix instruction where the two parts
// of k_attn.hip take two.  Q enters as binary16 scaled by a power of two per
// row (largest magnitude in [2^14, 2^15)): exact for elements down to 2^-28 of it.
// l sums the unrounded float32 w.
//
// A tail step (32 keys) is computed as in k_attn.hip: bfloat16 Q, K and V, the
// weights in two bfloat16 parts, the tree mask on the scores.
#include <math.h>

#include "sb_attn_device.h"
#include "sb_internal_fwd.h"

namespace sb {
namespace {

constexpr int kNW = 4;  // waves of a workgroup
constexpr int kT = 64 * kNW;

typedef _Float16 f16x2 __attribute__((ext_vector_type(2)));
typedef _Float16 f16x8 __attribute__((ext_vector_type(8)));
typedef float f32x2 __attribute__((ext_vector_type(2)));

__device__ __forceinline__ f32x4 mfma16h(f16x8 a, f16x8 b, f32x4 c) {
  return __builtin_amdgcn_mfma_f32_16x16x32_f16(a, b, c, 0, 0, 0);
}

__device__ __forceinline__ uint32_t pack_f16x2(float lo, float hi) {
  const f32x2 v = {lo, hi};
  return __builtin_bit_cast(uint32_t, __builtin_convertvector(v, f16x2));
}

// Four codes to binary16, exactly.
template <int FMT>
__device__ __forceinline__ void widen4(uint32_t w, uint32_t &lo, uint32_t &hi) {
  if (FMT == SB_KV_INT8) {
    // bytes of 0x64 over the code plus 128: the binary16 of 1024 + code + 128
    const f16x2 off = {(_Float16)1152.0f, (_Float16)1152.0f};
    const uint32_t a = __builtin_amdgcn_perm(w, 0x64646464u, 0x00050004u);
    const uint32_t b = __builtin_amdgcn_perm(w, 0x64646464u, 0x00070006u);
    lo = __builtin_bit_cast(uint32_t, __builtin_bit_cast(f16x2, a) - off);
    hi = __builtin_bit_cast(uint32_t, __builtin_bit_cast(f16x2, b) - off);
  } else {
    lo = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_f16_fp8((int)w, 1.0f, false));
    hi = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_f16_fp8((int)w, 1.0f, true));
  }
}
template <int FMT>
__device__ __forceinline__ f16x8 widen8(uint32_t w0, uint32_t w1) {
  uint4 o;
  widen4<FMT>(w0, o.x, o.y);
  widen4<FMT>(w1, o.z, o.w);
  return __builtin_bit_cast(f16x8, o);
}

// The largest of three (a NaN is passed over), one instruction; from fmaxf the
// compiler first makes quiet copies of its arguments.
__device__ __forceinline__ float max3(float a, float b, float c) {
  float r;
  asm("v_max3_f32 %0, %1, %2, %3" : "=v"(r) : "v"(a), "v"(b), "v"(c));
  return r;
}

__device__ __forceinline__ float lane_value(float v, int lane) {
  return __builtin_bit_cast(float, __builtin_amdgcn_readlane(__builtin_bit_cast(int, v), lane));
}

// The ancestor masks of the workgroup's rows into sanc: from the step's
// metadata where the caller has it, else from the tree, every row's at once in
// log2(n) rounds (a row takes over its jump's ancestors, then all jumps double).
// all: SB_MAX_ROWS masks of scratch; one thread per row.
static_assert(kT == SB_MAX_ROWS, "a thread per tree row");
template <int RT>
__device__ __forceinline__ void stage_masks(const QuantAttnArgs &a, const TreeArg &tree, int rb,
                                            int R, float inv_g, uint32_t (*sanc)[8],
                                            uint32_t (*all)[8]) {
  constexpr int RB = 16 * RT;
  __shared__ int16_t s_jump[SB_MAX_ROWS];
  if (!a.meta) {
    const int i = threadIdx.x;
    int jump = i < tree.n ? tree.parent[i] : -1;
    uint32_t on[8];
#pragma unroll
    for (int k = 0; k < 8; ++k) {
      on[k] = (i >> 5) == k ? 1u << (i & 31) : 0u;
      all[i][k] = on[k];
    }
    s_jump[i] = (int16_t)jump;
    __syncthreads();
    for (int step = 1; step < tree.n; step <<= 1) {
      const int next = jump >= 0 ? s_jump[jump] : -1;
      if (jump >= 0)
#pragma unroll
        for (int k = 0; k < 8; ++k) on[k] |= all[jump][k];
      __syncthreads();
      jump = next;
      s_jump[i] = (int16_t)next;
#pragma unroll
      for (int k = 0; k < 8; ++k) all[i][k] = on[k];
      __syncthreads();
    }
  }
  for (int i = threadIdx.x; i < RB * 8; i += kT) {
    const int r = rb * RB + (i >> 3), t = (int)(((float)r + 0.5f) * inv_g);
    sanc[i >> 3][i & 7] = r < R ? (a.meta ? a.meta->anc[t][i & 7] : all[t][i & 7]) : 0u;
  }
}

// D: head_dim; RT: 16-row query tiles of the workgroup.
template <int D, int FMT, int RT>
__global__ __launch_bounds__(kT, 2) void k_attn_quant(QuantAttnArgs a, TreeArg tree) {
  constexpr int KSD = D / 32;  // k-steps over head_dim (S)
  constexpr int NF = D / 16;   // fragments of K, or V, of a block; output tiles
  constexpr int RB = 16 * RT;
  constexpr int HD = D / 2;    // dimensions the waves' sums meet in at a time
  __shared__ __attribute__((aligned(16))) uint16_t sq[RB][D + 8];
  __shared__ float sqs[RB];  // score multiplier of a row, in units of log2
  __shared__ uint32_t sanc[RB][8];
  __shared__ float sm[kNW][RB], sl[kNW][RB];
  __shared__ __attribute__((aligned(16))) float so[kNW][RB][HD + 4];

  const int w = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int lane = threadIdx.x & 63;
  const int lr = lane & 15, lg = lane >> 4;
  const int G = a.n_heads / a.n_kv;
  const int R = a.n_tok * G;
  // Work unit (range, KV head, row block).  The row blocks of one range and head
  // follow each other on one XCD (workgroup b runs on XCD b % 8) and share its
  // reads through the L2; the tail's ranges, short ones, come first, so that what
  // does not fit the chip at once fills up behind them.
  const int turn = blockIdx.x >> 3;
  const int rb = turn % a.n_rb, unit = turn / a.n_rb * 8 + (blockIdx.x & 7);
  if (unit >= a.n_kv * a.n_chunks) return;
  const int g = unit % a.n_kv, split = unit / a.n_kv;
  const bool quant = split >= a.ct;
  const float c = a.scale * 1.44269504088896340736f;  // exp(x scale) = exp2(x c)

  // ---- an 8-bit range's first loads go out before anything waits: the wave's
  // first block, and the scales of its first 64 blocks, one per lane
  const int b0 = quant ? (int)((int64_t)a.n_blocks * (split - a.ct) / a.c8) : 0;
  const int b1 = quant ? (int)((int64_t)a.n_blocks * (split - a.ct + 1) / a.c8) : 0;
  const float *ks = a.k_scale + (size_t)g * a.cap_blocks, *vs = a.v_scale + (size_t)g * a.cap_blocks;
  const int bytes = a.cap_blocks * SB_KV_BLOCK * D;  // one head's codes: at most 2^27
  const __amdgpu_buffer_rsrc_t krs = uniform_rsrc(a.k8 + (size_t)g * bytes, bytes);
  const __amdgpu_buffer_rsrc_t vrs = uniform_rsrc(a.v8 + (size_t)g * bytes, bytes);
  i32x4 kf[NF], vf[NF];
  auto load = [&](i32x4 (&f)[NF], __amdgpu_buffer_rsrc_t rs, int b) {
    const int vo = b < b1 ? b * (SB_KV_BLOCK * D) + lane * 16 : bytes;
#pragma unroll
    for (int i = 0; i < NF; ++i) f[i] = __builtin_amdgcn_raw_buffer_load_b128(rs, vo, i * 1024, 0);
  };
  float kscales = 0.0f, vscales = 0.0f;
  auto load_scales = [&](int b) {
    const bool in = b + kNW * lane < b1;
    kscales = in ? ks[b + kNW * lane] : 0.0f;
    vscales = in ? vs[b + kNW * lane] : 0.0f;
  };
  if (quant) {
    load_scales(b0 + w);
    load(kf, krs, b0 + w);
    load(vf, vrs, b0 + w);
  }

  // ---- the rows' queries into LDS: binary16, scaled, or bfloat16 as they are
  constexpr int TPR = D / 8;  // threads per row
  constexpr int QPT = (RB * TPR + kT - 1) / kT;
  const float inv_g = 1.0f / (float)G;  // r / G = floor((r + 0.5) / G) for r < 2^20
  uint4 xq[QPT];
#pragma unroll
  for (int j = 0; j < QPT; ++j) {
    const int i = threadIdx.x + j * kT, r = rb * RB + i / TPR;
    const int t = (int)(((float)r + 0.5f) * inv_g);
    xq[j] = make_uint4(0, 0, 0, 0);
    if (i < RB * TPR && r < R)
      xq[j] = *(const uint4 *)((const uint16_t *)a.q +
                               ((size_t)t * a.n_heads + g * G + (r - t * G)) * D + (i % TPR) * 8);
  }
#pragma unroll
  for (int j = 0; j < QPT; ++j) {
    const int i = threadIdx.x + j * kT, rr = i / TPR, d0 = (i % TPR) * 8;
    if (i >= RB * TPR) break;  // whole waves
    uint4 x = xq[j];
    if (quant) {
      const uint32_t xw[4] = {x.x, x.y, x.z, x.w};
      uint32_t top = 0;
#pragma unroll
      for (int e = 0; e < 4; ++e) top = max(top, max(xw[e] & 0x7fffu, (xw[e] >> 16) & 0x7fffu));
#pragma unroll
      for (int o = TPR / 2; o > 0; o >>= 1) top = max(top, (uint32_t)__shfl_xor((int)top, o, 64));
      // 2^(14 - e) for a largest magnitude in [2^e, 2^(e + 1)), e >= -100
      int e = (int)(top >> 7) - 127;
      e = e < -100 ? -100 : e;
      const float f = __uint_as_float((uint32_t)(127 + 14 - e) << 23);
      uint4 o;
      o.x = pack_f16x2(bf2f((uint16_t)xw[0]) * f, bf2f((uint16_t)(xw[0] >> 16)) * f);
      o.y = pack_f16x2(bf2f((uint16_t)xw[1]) * f, bf2f((uint16_t)(xw[1] >> 16)) * f);
      o.z = pack_f16x2(bf2f((uint16_t)xw[2]) * f, bf2f((uint16_t)(xw[2] >> 16)) * f);
      o.w = pack_f16x2(bf2f((uint16_t)xw[3]) * f, bf2f((uint16_t)(xw[3] >> 16)) * f);
      x = o;
      if (d0 == 0) sqs[rr] = c * __uint_as_float((uint32_t)(127 + e - 14) << 23);
    } else if (d0 == 0) {
      sqs[rr] = c;
    }
    *(uint4 *)&sq[rr][d0] = x;
  }
  if (!quant) stage_masks<RT>(a, tree, rb, R, inv_g, sanc, (uint32_t (*)[8]) & so[0][0][0]);
  __syncthreads();

  f32x4 o[RT][NF];
  float m[RT], l[RT];
#pragma unroll
  for (int rt = 0; rt < RT; ++rt) {
#pragma unroll
    for (int dt = 0; dt < NF; ++dt) o[rt][dt] = f32x4{0.f, 0.f, 0.f, 0.f};
    m[rt] = -INFINITY;
    l[rt] = 0.0f;
  }
  // Row maxima nm: where one is larger than before, every sum so far scales down
  // to it (from -inf: to 0).  One branch for the row tiles together.
  auto raise = [&](float (&nm)[RT]) {
    bool more = false;
#pragma unroll
    for (int rt = 0; rt < RT; ++rt) more |= nm[rt] > m[rt];
    if (__ballot(more)) {
#pragma unroll
      for (int rt = 0; rt < RT; ++rt) {
        const float top = fmaxf(m[rt], nm[rt]);
        const float f = m[rt] == -INFINITY ? 0.0f : __builtin_amdgcn_exp2f(m[rt] - top);
        m[rt] = top;
        l[rt] *= f;
#pragma unroll
        for (int dt = 0; dt < NF; ++dt) o[rt][dt] *= f;
      }
    }
  };
  float unscale = 1.0f;  // of the wave's output sums

  if (quant) {
    float vtop = vscales;
    for (int b = b0 + w + kNW * (64 + lane); b < b1; b += kNW * 64) vtop = fmaxf(vtop, vs[b]);
    for (int i = 32; i > 0; i >>= 1) vtop = fmaxf(vtop, __shfl_xor(vtop, i, 64));
    vtop = fmaxf(vtop, 0x1p-100f);  // every V block zero, or as good as
    unscale = vtop * 0x1p-15f;
    const float rv = 0x1p15f / vtop;
    int at = 0;  // lane that holds the block's scales
    for (int b = b0 + w; b < b1; b += kNW) {
      // the query fragments are read again for every block: in registers over the
      // loop they would push others into memory
      asm volatile("" ::: "memory");
      if (at == 64) {
        load_scales(b);
        at = 0;
      }
      const float kscale = lane_value(kscales, at);
      // r = vscale 2^15 / vtop, no smaller than 2^-25 (a block whose codes then
      // count for less than 2^-40 of vtop each); a NaN stays
      float r = lane_value(vscales, at) * rv;
      r = r < 0x1p-25f ? 0x1p-25f : r;
      const float lr2 = __builtin_amdgcn_logf(r), ir = 1.0f / r;
      ++at;
      f32x4 s[RT][4];
#pragma unroll
      for (int rt = 0; rt < RT; ++rt)
#pragma unroll
        for (int kt = 0; kt < 4; ++kt) s[rt][kt] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int j = 0; j < KSD; ++j) {
        f16x8 qv[RT];
#pragma unroll
        for (int rt = 0; rt < RT; ++rt)
          qv[rt] = __builtin_bit_cast(f16x8, *(const uint4 *)&sq[rt * 16 + lr][32 * j + 8 * lg]);
#pragma unroll
        for (int kt = 0; kt < 4; ++kt) {
          const i32x4 f = kf[kt * (D / 64) + (j >> 1)];
          const f16x8 kv = widen8<FMT>((uint32_t)f[2 * (j & 1)], (uint32_t)f[2 * (j & 1) + 1]);
#pragma unroll
          for (int rt = 0; rt < RT; ++rt) s[rt][kt] = mfma16h(kv, qv[rt], s[rt][kt]);
        }
        // one k-step's query fragments at a time: with more of them early, RT = 3
        // has registers in memory, whose loads wait for the cache's
        if (RT == 3) __builtin_amdgcn_sched_barrier(0);
      }
      load(kf, krs, b + kNW);
      // ---- softmax: element e of s[rt][2 h + i] is key 32 h + 8 lg + 4 i + e
      f16x8 p[RT][2];
      float ck[RT], nm[RT];
#pragma unroll
      for (int rt = 0; rt < RT; ++rt) {
        float mx = fmaxf(s[rt][0][0], s[rt][0][1]);
#pragma unroll
        for (int e = 2; e < 16; e += 2) mx = max3(mx, s[rt][e >> 2][e & 3], s[rt][e >> 2][(e & 3) + 1]);
        ck[rt] = sqs[rt * 16 + lr] * kscale;
        nm[rt] = max_x32(max_x16(mx)) * ck[rt];
      }
      raise(nm);
#pragma unroll
      for (int rt = 0; rt < RT; ++rt) {
        const float base = lr2 - (m[rt] == -INFINITY ? 0.0f : m[rt]);
        float ps = 0.0f;
#pragma unroll
        for (int h = 0; h < 2; ++h) {
          float x[8];
#pragma unroll
          for (int e = 0; e < 8; ++e) {
            x[e] = __builtin_amdgcn_exp2f(fmaf(s[rt][2 * h + (e >> 2)][e & 3], ck[rt], base));
            ps += x[e];
          }
          uint4 pk;
          pk.x = pack_f16x2(x[0], x[1]);
          pk.y = pack_f16x2(x[2], x[3]);
          pk.z = pack_f16x2(x[4], x[5]);
          pk.w = pack_f16x2(x[6], x[7]);
          p[rt][h] = __builtin_bit_cast(f16x8, pk);
        }
        l[rt] = fmaf(ps, ir, l[rt]);
        if (RT == 3) __builtin_amdgcn_sched_barrier(0);
      }
#pragma unroll
      for (int dt = 0; dt < NF; ++dt)
#pragma unroll
        for (int h = 0; h < 2; ++h) {
          const f16x8 vv = widen8<FMT>((uint32_t)vf[dt][2 * h], (uint32_t)vf[dt][2 * h + 1]);
#pragma unroll
          for (int rt = 0; rt < RT; ++rt) o[rt][dt] = mfma16h(vv, p[rt][h], o[rt][dt]);
        }
      load(vf, vrs, b + kNW);
    }
  } else {
    const int nkeys = a.tail_len + a.n_tok, n_steps = (nkeys + 31) >> 5, ts = split;
    const int st0 = n_steps * ts / a.ct, st1 = n_steps * (ts + 1) / a.ct;
    const int bytes = a.tail_cap * D * 2;
    const __amdgpu_buffer_rsrc_t krs = uniform_rsrc(a.tk + (size_t)g * a.tail_cap * D, bytes);
    const __amdgpu_buffer_rsrc_t vrs = uniform_rsrc(a.tv + (size_t)g * a.tail_cap * D, bytes);
    for (int st = st0 + w; st < st1; st += kNW) {
      const int k0 = st * 32 + 8 * lg;  // this lane's 8 keys
      i32x4 kf[2][KSD], vf[NF];
      // row rho of key tile i is key 8 (rho / 4) + 4 i + rho % 4; slots past
      // nkeys read zero
#pragma unroll
      for (int i = 0; i < 2; ++i) {
        const int slot = st * 32 + 8 * (lr >> 2) + 4 * i + (lr & 3);
        const int vo = slot < nkeys ? (slot * D + 8 * lg) * 2 : bytes;
#pragma unroll
        for (int j = 0; j < KSD; ++j) kf[i][j] = __builtin_amdgcn_raw_buffer_load_b128(krs, vo, j * 64, 0);
      }
#pragma unroll
      for (int dt = 0; dt < NF; ++dt)
        vf[dt] = __builtin_amdgcn_raw_buffer_load_b128(
            vrs, k0 < nkeys ? ((16 * dt + lr) * a.tail_cap + k0) * 2 : bytes, 0, 0);
      f32x4 s[RT][2];
#pragma unroll
      for (int rt = 0; rt < RT; ++rt) {
        s[rt][0] = s[rt][1] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int j = 0; j < KSD; ++j) {
          const bf16x8 qv = as_bf16x8(*(const uint4 *)&sq[rt * 16 + lr][32 * j + 8 * lg]);
#pragma unroll
          for (int i = 0; i < 2; ++i)
            s[rt][i] = mfma16(__builtin_bit_cast(bf16x8, kf[i][j]), qv, s[rt][i]);
        }
      }
      if (k0 + 8 > nkeys) {  // slots never written count as zero in V too (0 x NaN)
        const int valid = nkeys - k0;
#pragma unroll
        for (int dt = 0; dt < NF; ++dt)
#pragma unroll
          for (int e = 0; e < 4; ++e)
            vf[dt][e] &= (int)((2 * e < valid ? 0x0000ffffu : 0u) | (2 * e + 1 < valid ? 0xffff0000u : 0u));
      }
      float nm[RT];
#pragma unroll
      for (int rt = 0; rt < RT; ++rt) {
        const uint32_t vis = visible8(sanc[rt * 16 + lr], k0, a.tail_len, nkeys);
        float mx = -INFINITY;
#pragma unroll
        for (int e = 0; e < 8; ++e) {
          const float x = (vis >> e) & 1u ? s[rt][e >> 2][e & 3] : -INFINITY;
          s[rt][e >> 2][e & 3] = x;
          mx = fmaxf(mx, x);
        }
        nm[rt] = max_x32(max_x16(mx)) * c;
      }
      raise(nm);
#pragma unroll
      for (int rt = 0; rt < RT; ++rt) {
        const float mc = m[rt] == -INFINITY ? 0.0f : m[rt];
        float x[8];
        float ps = 0.0f;
        uint32_t hi[4], lo[4];
#pragma unroll
        for (int e = 0; e < 8; ++e) {
          x[e] = __builtin_amdgcn_exp2f(fmaf(s[rt][e >> 2][e & 3], c, -mc));  // exp2(-inf) = 0 when masked
          ps += x[e];
        }
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          hi[e] = pack_bf16x2(x[2 * e], x[2 * e + 1]);
          // p - bf16(p) is exact in float32
          lo[e] = pack_bf16x2(x[2 * e] - __uint_as_float(hi[e] << 16),
                              x[2 * e + 1] - __uint_as_float(hi[e] & 0xffff0000u));
        }
        l[rt] += ps;
        const bf16x8 ph = as_bf16x8(make_uint4(hi[0], hi[1], hi[2], hi[3]));
        const bf16x8 pl = as_bf16x8(make_uint4(lo[0], lo[1], lo[2], lo[3]));
#pragma unroll
        for (int dt = 0; dt < NF; ++dt) {
          o[rt][dt] = mfma16(__builtin_bit_cast(bf16x8, vf[dt]), ph, o[rt][dt]);
          o[rt][dt] = mfma16(__builtin_bit_cast(bf16x8, vf[dt]), pl, o[rt][dt]);
        }
      }
    }
  }

  // ---- the waves' sums, in wave order, against the largest maximum; HD
  // dimensions at a time
#pragma unroll
  for (int rt = 0; rt < RT; ++rt) {
    const float sum = sum_x32(sum_x16(l[rt]));
    if (lg == 0) {
      sm[w][rt * 16 + lr] = m[rt];
      sl[w][rt * 16 + lr] = sum;
    }
  }
  __syncthreads();
#pragma unroll
  for (int rt = 0; rt < RT; ++rt) {
    float M = sm[0][rt * 16 + lr];
#pragma unroll
    for (int v = 1; v < kNW; ++v) M = fmaxf(M, sm[v][rt * 16 + lr]);
    const float f = m[rt] == -INFINITY ? 0.0f : __builtin_amdgcn_exp2f(m[rt] - M) * unscale;
#pragma unroll
    for (int dt = 0; dt < NF; ++dt) o[rt][dt] *= f;
  }
  const size_t base = ((size_t)g * a.n_chunks + split) * R;
#pragma unroll
  for (int half = 0; half < 2; ++half) {
    if (half) __syncthreads();
#pragma unroll
    for (int rt = 0; rt < RT; ++rt)
#pragma unroll
      for (int dt = 0; dt < NF / 2; ++dt)
        *(f32x4 *)&so[w][rt * 16 + lr][16 * dt + 4 * lg] = o[rt][half * (NF / 2) + dt];
    __syncthreads();
    for (int i = threadIdx.x; i < RB * (HD / 4); i += kT) {
      const int rr = i / (HD / 4), d0 = (i % (HD / 4)) * 4, r = rb * RB + rr;
      f32x4 x = *(const f32x4 *)&so[0][rr][d0];
#pragma unroll
      for (int v = 1; v < kNW; ++v) x += *(const f32x4 *)&so[v][rr][d0];
      if (r < R) *(f32x4 *)&a.part_o[(base + r) * D + half * HD + d0] = x;
    }
  }
  if (threadIdx.x < RB) {
    const int rr = threadIdx.x, r = rb * RB + rr;
    float M = sm[0][rr], L = 0.0f;
#pragma unroll
    for (int v = 1; v < kNW; ++v) M = fmaxf(M, sm[v][rr]);
#pragma unroll
    for (int v = 0; v < kNW; ++v)
      if (sm[v][rr] != -INFINITY) L += sl[v][rr] * __builtin_amdgcn_exp2f(sm[v][rr] - M);
    // the merge takes the maximum in units of the natural exponent
    if (r < R) *(float2 *)&a.part_ml[(base + r) * 2] = make_float2(M * 0.69314718055994530942f, L);
  }
}

template <int D, int FMT>
hipError_t launch_rt(const QuantAttnArgs &a, const TreeArg &tree, int rt, hipStream_t s) {
  const dim3 grid(round_up(a.n_kv * a.n_chunks, 8) * a.n_rb), block(kT);
  switch (rt) {
    case 1: hipLaunchKernelGGL((k_attn_quant<D, FMT, 1>), grid, block, 0, s, a, tree); break;
    case 2: hipLaunchKernelGGL((k_attn_quant<D, FMT, 2>), grid, block, 0, s, a, tree); break;
    case 3: hipLaunchKernelGGL((k_attn_quant<D, FMT, 3>), grid, block, 0, s, a, tree); break;
    default: return hipErrorInvalidValue;
  }
  return hipGetLastError();
}

}  // namespace

// Row tiles of a workgroup: as few row blocks as three tiles a wave allow.
// Ranges: two workgroups per compute unit, shared between the blocks and the
// tail by their steps (a tail step of 32 keys reads what a block of 64 does),
// at most one range per four steps, so that every wave has one.
QuantAttnPlan quant_attn_plan(int n_kv, int n_blocks, int tail_keys, int rows) {
  QuantAttnPlan p{};
  const int tiles = ceil_div(rows, 16), steps = ceil_div(tail_keys, 32);
  p.n_rb = ceil_div(tiles, kQuantMaxRowTiles);
  p.rt = ceil_div(tiles, p.n_rb);
  int per = kQuantTargetGroups / (n_kv * p.n_rb);
  if (per > kQuantMaxRanges) per = kQuantMaxRanges;
  if (per < 2) per = 2;
  p.ct = (int)((int64_t)per * steps / (n_blocks + steps));
  if (p.ct > ceil_div(steps, kNW)) p.ct = ceil_div(steps, kNW);
  if (p.ct < 1) p.ct = 1;
  p.c8 = per - (p.ct > 1 ? p.ct : 0);
  if (p.c8 > ceil_div(n_blocks, kNW)) p.c8 = ceil_div(n_blocks, kNW);
  if (p.c8 < 1 && n_blocks > 0) p.c8 = 1;
  return p;
}

hipError_t launch_attn_quant(const QuantAttnArgs &args, const TreeArg &tree, hipStream_t s) {
  QuantAttnArgs a = args;
  const QuantAttnPlan p =
      quant_attn_plan(a.n_kv, a.n_blocks, a.tail_len + a.n_tok, a.n_tok * (a.n_heads / a.n_kv));
  if (a.n_chunks != p.c8 + p.ct || a.n_tok < 1) return hipErrorInvalidValue;
  a.c8 = p.c8;
  a.ct = p.ct;
  a.n_rb = p.n_rb;
  if (a.head_dim == 128)
    return a.format == SB_KV_INT8 ? launch_rt<128, SB_KV_INT8>(a, tree, p.rt, s)
                                  : launch_rt<128, SB_KV_E4M3>(a, tree, p.rt, s);
  if (a.head_dim == 64)
    return a.format == SB_KV_INT8 ? launch_rt<64, SB_KV_INT8>(a, tree, p.rt, s)
                                  : launch_rt<64, SB_KV_E4M3>(a, tree, p.rt, s);
  return hipErrorInvalidValue;
}

}  // namespace sb
