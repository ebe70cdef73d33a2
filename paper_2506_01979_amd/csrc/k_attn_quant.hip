// Branch-masked attention over a prefix cache held in 8 bits, with a 16-bit
// tail behind it (the committed tokens that fill no block yet, then the
// tree's rows): the attention of k_attn.hip, one softmax over both parts.
//
// Flash-decoding split as there: the steps of every KV head -- its blocks of 64
// keys, then steps of 32 tail keys -- are cut into ranges of one weight, one
// workgroup each (and per block of at most 48 query rows), and the merge kernels
// of k_attn.hip combine the ranges.  The four waves share a range's steps, every
// fourth each, with a running softmax for all of the workgroup's rows: no barrier
// in the loop, every code is converted once per row block, and the waves' sums
// meet in LDS after the last step.  (Waves that share the rows instead, with the
// steps in a ring of LDS buffers, met at a barrier a step and read every fragment
// once per wave: 81 us where this form took 49, 13B, 129 rows, prefix 8192, both with
// weights of one part.)
//
// What bounds it.  Few rows: the launch, the first loads' latency and the merge
// (68M, 1 row, 300 keys: 5.7 + 2.5 us for 1 MB; 70B, 1 row, 32773 keys: 15.5 + 4 us
// where the 67 MB alone take 14).  Many rows: the vector and the matrix unit, which
// two waves a SIMD hardly overlap -- 510 (int8 638) and 144 instructions a block with
// three row tiles; 13B, 129 rows, prefix 8192: busy for 59 and 35 of the 98 kcycles
// that a wave lives, 57 us with the merge.
//
// An 8-bit block (64 keys): its codes come in operand order, 16 bytes per lane
// and fragment, straight into registers, and are widened to binary16 there,
// where both formats are exact: int8 by placing the byte under the exponent of
// 1024 and subtracting 1152, e4m3 by the conversion instruction.  The scales
// never touch the codes: K's multiplies the scores with the softmax factor, V's
// multiplies the softmax weights,
//   S^T = K Q^T;  w = exp2(s kscale c - m + log2 r);  l += w / r;  O^T += V^T w^T,
//   r = vscale 2^15 / (the largest vscale of the wave's blocks),
// so that w <= 2^15 in two binary16 parts, a product each, keeps 22 bits, down to steps
// of 2^-40 of the largest weight: no less than the two bfloat16 parts of k_attn.hip.
// (One part, 11 bits, moves 9 % of the bfloat16 outputs by a step; 13B, 129 rows,
// prefix 8192 49.6 us with it, 57.0 with two; 7B, 33 rows 14.2 and 14.4.)  Q enters as
// binary16 scaled by a power of two per row (largest magnitude in [2^14, 2^15)): exact
// for elements down to 2^-28 of it.
// l sums the unrounded float32 w.
//
// A tail step (32 keys) is computed as in k_attn.hip: bfloat16 Q, K and V, the
// weights in two bfloat16 parts, the tree mask on the scores.  A wave takes its
// tail steps before its blocks, so that their loads go out with the launch.
#include <math.h>

#include "sb_attn_device.h"
#include "sb_internal_fwd.h"

namespace sb {
namespace {

typedef _Float16 f16x2 __attribute__((ext_vector_type(2)));
typedef _Float16 f16x8 __attribute__((ext_vector_type(8)));
typedef float f32x2 __attribute__((ext_vector_type(2)));
typedef uint16_t u16x2 __attribute__((ext_vector_type(2)));

constexpr int kNW = 4;  // waves of a workgroup
constexpr int kT = 64 * kNW;
constexpr int kTailWeight = 3;

// A tree as a kernel argument: its parents, and up to kMaskArgRows rows' ancestor
// masks (2 KB of the 4 that arguments have).
constexpr int kMaskArgRows = 128;
struct TreeMasks {
  int16_t parent[SB_MAX_ROWS];
  uint32_t mask[kMaskArgRows][4];
};

__device__ __forceinline__ f32x4 mfma16h(f16x8 a, f16x8 b, f32x4 c) {
  return __builtin_amdgcn_mfma_f32_16x16x32_f16(a, b, c, 0, 0, 0);
}

__device__ __forceinline__ uint32_t pack_f16x2(float lo, float hi) {
  const f32x2 v = {lo, hi};
  return __builtin_bit_cast(uint32_t, __builtin_convertvector(v, f16x2));
}

// Eight floats in [0, 2^15] as two binary16 parts, 22 bits of each down to 2^-24.
__device__ __forceinline__ void split_f16(const float (&x)[8], f16x8 &hi, f16x8 &lo) {
  // a factor that the compiler does not know, so that widening, (exact) difference
  // and rounding stay one instruction
  float minus = -1.0f;
  asm("" : "+s"(minus));
#pragma unroll
  for (int e = 0; e < 8; e += 2) {
    const f16x2 h = __builtin_convertvector(f32x2{x[e], x[e + 1]}, f16x2);
    hi[e] = h[0];
    hi[e + 1] = h[1];
    lo[e] = (_Float16)fmaf((float)h[0], minus, x[e]);
    lo[e + 1] = (_Float16)fmaf((float)h[1], minus, x[e + 1]);
  }
}

// All ones in the halves of w that are not finite as bfloat16.
__device__ __forceinline__ uint32_t not_finite(int w) {
  return ((w & 0x7f80) == 0x7f80 ? 0xffffu : 0u) | ((w & 0x7f800000) == 0x7f800000 ? 0xffff0000u : 0u);
}
// Whether any value of a wave's fragments is; they are then zeros.
template <int N>
__device__ __forceinline__ bool take_not_finite(i32x4 (&f)[N]) {
  u16x2 top = {0, 0};
#pragma unroll
  for (int i = 0; i < N; ++i)
#pragma unroll
    for (int e = 0; e < 4; ++e)
      top = __builtin_elementwise_max(top, __builtin_bit_cast(u16x2, f[i][e] & 0x7fff7fff));
  if (!__ballot(top[0] >= 0x7f80 || top[1] >= 0x7f80)) return false;
#pragma unroll
  for (int i = 0; i < N; ++i)
#pragma unroll
    for (int e = 0; e < 4; ++e) f[i][e] &= (int)~not_finite(f[i][e]);
  return true;
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

// The larger (a NaN is passed over) in one instruction: from fmaxf the compiler
// first makes quiet copies of arguments that it did not compute itself.
__device__ __forceinline__ float max2(float a, float b) {
  return __builtin_amdgcn_fmed3f(a, b, INFINITY);
}

__device__ __forceinline__ float lane_value(float v, int lane) {
  return __builtin_bit_cast(float, __builtin_amdgcn_readlane(__builtin_bit_cast(int, v), lane));
}

// What a launch's workgroup works on: a range of a KV head's steps -- its 8-bit
// blocks [b0, b1) and steps [t0, t1) of 32 tail keys -- for one block of rows.
struct Range {
  int g, split, rb, b0, b1, t0, t1;
  bool live;
};
// The row blocks of one range and head follow each other on one XCD (workgroup
// b runs on XCD b % 8) and share its reads through the L2.  The blocks, then the
// tail, in ranges of one weight: a tail step takes about as long as kTailWeight
// blocks (its weights go through two products, its scores through the mask).
__device__ __forceinline__ Range range_of(const QuantAttnArgs &a) {
  Range r;
  const int turn = blockIdx.x >> 3, unit = turn / a.n_rb * 8 + (blockIdx.x & 7);
  r.rb = turn % a.n_rb;
  r.live = unit < a.n_kv * a.n_chunks;
  r.g = unit % a.n_kv;
  r.split = unit / a.n_kv;
  const int steps = (a.tail_len + a.n_tok + 31) >> 5, all = a.n_blocks + kTailWeight * steps;
  const int u0 = (int)((int64_t)all * r.split / a.n_chunks);
  const int u1 = (int)((int64_t)all * (r.split + 1) / a.n_chunks);
  r.b0 = min(u0, a.n_blocks);
  r.b1 = min(u1, a.n_blocks);
  r.t0 = max(u0 - a.n_blocks, 0) / kTailWeight;
  r.t1 = max(u1 - a.n_blocks, 0) / kTailWeight;
  return r;
}

// The ancestor masks of the tree's rows, as two 16-byte words each, into `on`:
// from the step's metadata or the launch's arguments where they have them (up to
// kMaskArgRows rows), else from the tree, every row's at once in log2(n) rounds (a
// row takes over its jump's ancestors, then all jumps double; 4 us for 129 rows,
// where the arguments take 1).  on and tmp: SB_MAX_ROWS masks each in LDS.
__device__ void stage_masks(const QuantAttnArgs &a, const TreeMasks &tree, uint4 (*on)[2],
                            uint4 (*tmp)[2]) {
  __shared__ int16_t s_jump[2][SB_MAX_ROWS];
  const int n = a.n_tok, nt = blockDim.x;
  if (a.meta) {
    for (int i = threadIdx.x; i < n * 2; i += nt) on[i >> 1][i & 1] = ((const uint4 *)a.meta->anc[i >> 1])[i & 1];
    __syncthreads();
    return;
  }
  if (n <= kMaskArgRows) {
    for (int i = threadIdx.x; i < n; i += nt) {
      on[i][0] = make_uint4(tree.mask[i][0], tree.mask[i][1], tree.mask[i][2], tree.mask[i][3]);
      on[i][1] = make_uint4(0, 0, 0, 0);
    }
    __syncthreads();
    return;
  }
  for (int i = threadIdx.x; i < n; i += nt) {
    const uint32_t bit = 1u << (i & 31);
    const int k = i >> 5;
    on[i][0] = make_uint4(k == 0 ? bit : 0u, k == 1 ? bit : 0u, k == 2 ? bit : 0u, k == 3 ? bit : 0u);
    on[i][1] = make_uint4(k == 4 ? bit : 0u, k == 5 ? bit : 0u, k == 6 ? bit : 0u, k == 7 ? bit : 0u);
    s_jump[0][i] = tree.parent[i];
  }
  __syncthreads();
  uint4(*from)[2] = on, (*to)[2] = tmp;
  int turn = 0;
  for (int step = 1; step < n; step <<= 1) {
    for (int i = threadIdx.x; i < n; i += nt) {
      const int jump = s_jump[turn][i], j = jump >= 0 ? jump : i;
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        const uint4 x = from[i][h], y = from[j][h];
        to[i][h] = make_uint4(x.x | y.x, x.y | y.y, x.z | y.z, x.w | y.w);
      }
      s_jump[turn ^ 1][i] = jump >= 0 ? s_jump[turn][jump] : (int16_t)-1;
    }
    __syncthreads();
    uint4(*swap)[2] = from;
    from = to;
    to = swap;
    turn ^= 1;
  }
  if (from != on) {
    for (int i = threadIdx.x; i < n * 2; i += nt) on[i >> 1][i & 1] = from[i >> 1][i & 1];
    __syncthreads();
  }
}

// Eight bfloat16 of a query row as binary16 times 2^(14 - e), e the exponent of
// the row's largest magnitude (bits top), at least -100; mult: what a score
// against them must be multiplied by, c 2^(e - 14).
__device__ __forceinline__ uint4 scale_query(uint4 x, uint32_t top, float c, float &mult) {
  int e = (int)(top >> 7) - 127;
  e = e < -100 ? -100 : e;
  const float f = __uint_as_float((uint32_t)(127 + 14 - e) << 23);
  mult = c * __uint_as_float((uint32_t)(127 + e - 14) << 23);
  const uint32_t w[4] = {x.x, x.y, x.z, x.w};
  uint32_t o[4];
#pragma unroll
  for (int i = 0; i < 4; ++i)
    o[i] = pack_f16x2(bf2f((uint16_t)w[i]) * f, bf2f((uint16_t)(w[i] >> 16)) * f);
  return make_uint4(o[0], o[1], o[2], o[3]);
}
__device__ __forceinline__ uint32_t largest_bits(uint4 x) {
  const uint32_t w[4] = {x.x, x.y, x.z, x.w};
  uint32_t top = 0;
#pragma unroll
  for (int i = 0; i < 4; ++i) top = max(top, max(w[i] & 0x7fffu, (w[i] >> 16) & 0x7fffu));
  return top;
}

// The scales of up to 64 blocks, one per lane: block b0 + stride lane.
struct Scales {
  float k, v;
  __device__ __forceinline__ void load(const QuantAttnArgs &a, int g, int b, int stride, int b1) {
    const int at = b + stride * (int)(threadIdx.x & 63);
    const bool in = at < b1;
    k = in ? a.k_scale[(size_t)g * a.cap_blocks + at] : 0.0f;
    v = in ? a.v_scale[(size_t)g * a.cap_blocks + at] : 0.0f;
  }
  // The largest V scale of every stride-th block of [b, b1), at least 2^-100
  // (every V block zero, or as good as).
  __device__ __forceinline__ float largest_v(const QuantAttnArgs &a, int g, int b, int stride,
                                             int b1) const {
    float top = v;
    for (int at = b + stride * (64 + (int)(threadIdx.x & 63)); at < b1; at += stride * 64)
      top = fmaxf(top, a.v_scale[(size_t)g * a.cap_blocks + at]);
    for (int i = 32; i > 0; i >>= 1) top = fmaxf(top, __shfl_xor(top, i, 64));
    return fmaxf(top, 0x1p-100f);
  }
};
// A block's factors from its scales, rv = 2^15 / (the largest V scale): r no
// smaller than 2^-25 (a block whose codes then count for less than 2^-40 of the
// largest scale each); a NaN stays.
struct BlockScale {
  float k, lr2, ir;  // K's scale, log2 r, 1 / r
  __device__ __forceinline__ BlockScale(const Scales &s, int lane, float rv) {
    k = lane_value(s.k, lane);
    float r = lane_value(s.v, lane) * rv;
    r = r < 0x1p-25f ? 0x1p-25f : r;
    lr2 = __builtin_amdgcn_logf(r);
    ir = 1.0f / r;
  }
};

// RT row tiles of one wave: output sums, maxima (log2 units) and sums of the
// softmax.  Lane (lr, lg): row lr of every tile, dimensions 16 dt + 4 lg .. + 3.
// TIGHT: the fragments come out of LDS as they are needed, a k-step or an output
// tile at a time -- with more of them early, registers end up in memory, whose
// loads then wait for the cache's.
template <int D, int FMT, int RT, bool TIGHT>
struct Tiles {
  static constexpr int KSD = D / 32;  // k-steps over head_dim (S)
  static constexpr int NF = D / 16;   // fragments of K, or V, of a step; output tiles
  f32x4 o[RT][NF];
  float m[RT], l[RT];
  __device__ __forceinline__ void init() {
#pragma unroll
    for (int rt = 0; rt < RT; ++rt) {
#pragma unroll
      for (int dt = 0; dt < NF; ++dt) o[rt][dt] = f32x4{0.f, 0.f, 0.f, 0.f};
      m[rt] = -INFINITY;
      l[rt] = 0.0f;
    }
  }
  __device__ __forceinline__ void scale_out(float f) {
#pragma unroll
    for (int rt = 0; rt < RT; ++rt)
#pragma unroll
      for (int dt = 0; dt < NF; ++dt) o[rt][dt] *= f;
  }
  // The largest finite one: an infinity in the tail's V stays in its own sums.
  __device__ __forceinline__ float largest_out() const {
    float top = 0.0f;
#pragma unroll
    for (int rt = 0; rt < RT; ++rt)
#pragma unroll
      for (int dt = 0; dt < NF; ++dt)
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          const float x = fabsf(o[rt][dt][e]);
          top = fmaxf(top, x < INFINITY ? x : 0.0f);
        }
    for (int i = 32; i > 0; i >>= 1) top = fmaxf(top, __shfl_xor(top, i, 64));
    return top;
  }
  // Row maxima nm: where one is larger than before, every sum so far scales down
  // to it (from -inf: to 0).  One branch for the row tiles together.
  __device__ __forceinline__ void raise(const float (&nm)[RT]) {
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
  }
  // One 8-bit block.  q(rt, j): query fragment of k-step j; kfrag(i), vfrag(i):
  // the block's fragments; cq(rt): the rows' score multiplier; scored(): called
  // once K is used up.
  template <class Q, class KF, class VF, class C, class S>
  __device__ __forceinline__ void block(const Q &q, const KF &kfrag, const VF &vfrag, const C &cq,
                                        const BlockScale &bs, const S &scored) {
    f32x4 s[RT][4];
#pragma unroll
    for (int rt = 0; rt < RT; ++rt)
#pragma unroll
      for (int kt = 0; kt < 4; ++kt) s[rt][kt] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int j = 0; j < KSD; ++j) {
      f16x8 qv[RT];
#pragma unroll
      for (int rt = 0; rt < RT; ++rt) qv[rt] = q(rt, j);
#pragma unroll
      for (int kt = 0; kt < 4; ++kt) {
        const uint2 f = kfrag(kt * (D / 64) + (j >> 1), j & 1);
        const f16x8 kv = widen8<FMT>(f.x, f.y);
#pragma unroll
        for (int rt = 0; rt < RT; ++rt) s[rt][kt] = mfma16h(kv, qv[rt], s[rt][kt]);
      }
      if (TIGHT) __builtin_amdgcn_sched_barrier(0);
    }
    scored();
    // element e of s[rt][2 h + i] is key 32 h + 8 lg + 4 i + e
    float ck[RT], nm[RT];
#pragma unroll
    for (int rt = 0; rt < RT; ++rt) {
      float mx = max2(max2(max2(s[rt][0][0], s[rt][0][1]), max2(s[rt][0][2], s[rt][0][3])),
                      max2(max2(s[rt][1][0], s[rt][1][1]), max2(s[rt][1][2], s[rt][1][3])));
      mx = max2(mx, max2(max2(max2(s[rt][2][0], s[rt][2][1]), max2(s[rt][2][2], s[rt][2][3])),
                         max2(max2(s[rt][3][0], s[rt][3][1]), max2(s[rt][3][2], s[rt][3][3]))));
      ck[rt] = cq(rt) * bs.k;
      nm[rt] = max_x32(max_x16(mx)) * ck[rt];
    }
    raise(nm);
    // 32 keys at a time: the weights of the second half beside the products of the first
    float ps[RT];
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      f16x8 hi[RT], lo[RT];
#pragma unroll
      for (int rt = 0; rt < RT; ++rt) {
        const float base = bs.lr2 - (m[rt] == -INFINITY ? 0.0f : m[rt]);
        float x[8];
        if (h == 0) ps[rt] = 0.0f;
#pragma unroll
        for (int e = 0; e < 8; ++e) {
          x[e] = __builtin_amdgcn_exp2f(fmaf(s[rt][2 * h + (e >> 2)][e & 3], ck[rt], base));
          ps[rt] += x[e];
        }
        split_f16(x, hi[rt], lo[rt]);
        if (h == 1) l[rt] = fmaf(ps[rt], bs.ir, l[rt]);
        if (TIGHT) __builtin_amdgcn_sched_barrier(0);
      }
#pragma unroll
      for (int dt = 0; dt < NF; ++dt) {
        const uint2 f = vfrag(dt, h);
        const f16x8 vv = widen8<FMT>(f.x, f.y);
#pragma unroll
        for (int rt = 0; rt < RT; ++rt) o[rt][dt] = mfma16h(vv, hi[rt], o[rt][dt]);
#pragma unroll
        for (int rt = 0; rt < RT; ++rt) o[rt][dt] = mfma16h(vv, lo[rt], o[rt][dt]);
        if (TIGHT && (dt & 1)) __builtin_amdgcn_sched_barrier(0);
      }
    }
  }
  // NaN into the sums of dimension tile dt of every row that sees (vis(rt)) a key
  // whose value in V's fragment is not finite.
  template <class V>
  __device__ __forceinline__ void show_not_finite(int dt, i32x4 v, const V &vis) {
    i32x4 bad;
#pragma unroll
    for (int e = 0; e < 4; ++e) bad[e] = (int)(not_finite(v[e]) & 0x3f803f80u);  // ones
    if (!__ballot((bad[0] | bad[1] | bad[2] | bad[3]) != 0)) return;
#pragma unroll
    for (int rt = 0; rt < RT; ++rt) {
      const uint32_t see = vis(rt);
      i32x4 one;
#pragma unroll
      for (int e = 0; e < 4; ++e)
        one[e] = (int)(((see >> (2 * e)) & 1u ? 0x3f80u : 0u) | ((see >> (2 * e + 1)) & 1u ? 0x3f800000u : 0u));
      const f32x4 n = mfma16(__builtin_bit_cast(bf16x8, bad), __builtin_bit_cast(bf16x8, one),
                             f32x4{0.f, 0.f, 0.f, 0.f});
#pragma unroll
      for (int e = 0; e < 4; ++e) o[rt][dt][e] = n[e] > 0.0f ? NAN : o[rt][dt][e];
    }
  }
  // One step of 32 tail keys.  q(rt, j): bfloat16 query fragment; kfrag(i, j):
  // key tile i, k-step j; vfrag(dt); vis(rt): bit e of it, key 8 lg + e of the
  // step is visible to the lane's row.
  template <class Q, class KF, class VF, class V, class S>
  __device__ __forceinline__ void tail(const Q &q, const KF &kfrag, const VF &vfrag, const V &vis,
                                       float c, const S &scored) {
    f32x4 s[RT][2];
#pragma unroll
    for (int rt = 0; rt < RT; ++rt) s[rt][0] = s[rt][1] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int j = 0; j < KSD; ++j)
#pragma unroll
      for (int i = 0; i < 2; ++i) {
        const bf16x8 kv = kfrag(i, j);
#pragma unroll
        for (int rt = 0; rt < RT; ++rt) s[rt][i] = mfma16(kv, q(rt, j), s[rt][i]);
        if (TIGHT) __builtin_amdgcn_sched_barrier(0);
      }
    scored();
    float nm[RT];
#pragma unroll
    for (int rt = 0; rt < RT; ++rt) {
      const uint32_t see = vis(rt);
      float mx = -INFINITY;
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        const float x = (see >> e) & 1u ? s[rt][e >> 2][e & 3] : -INFINITY;
        s[rt][e >> 2][e & 3] = x;
        mx = fmaxf(mx, x);
      }
      nm[rt] = max_x32(max_x16(mx)) * c;
    }
    raise(nm);
    bf16x8 ph[RT], pl[RT];
#pragma unroll
    for (int rt = 0; rt < RT; ++rt) {
      const float mc = m[rt] == -INFINITY ? 0.0f : m[rt];
      float x[8], ps = 0.0f;
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
      ph[rt] = as_bf16x8(make_uint4(hi[0], hi[1], hi[2], hi[3]));
      pl[rt] = as_bf16x8(make_uint4(lo[0], lo[1], lo[2], lo[3]));
      if (TIGHT) __builtin_amdgcn_sched_barrier(0);
    }
#pragma unroll
    for (int dt = 0; dt < NF; ++dt) {
      const bf16x8 v = vfrag(dt);
#pragma unroll
      for (int rt = 0; rt < RT; ++rt) o[rt][dt] = mfma16(v, ph[rt], o[rt][dt]);
#pragma unroll
      for (int rt = 0; rt < RT; ++rt) o[rt][dt] = mfma16(v, pl[rt], o[rt][dt]);
      if (TIGHT && (dt & 1)) __builtin_amdgcn_sched_barrier(0);
    }
  }
};

// Which of the 8 tail keys from k0 (a multiple of 8) a row with ancestor mask
// anc sees, as visible8 of k_attn.hip but without branches.
__device__ __forceinline__ uint32_t tail_visible(const uint32_t *anc, int k0, int tail_len, int nkeys) {
  const int jt = k0 - tail_len, at = max(jt, 0), pre = min(max(-jt, 0), 8);
  const int wi = min(at >> 5, 7);
  const uint64_t win = (uint64_t)anc[wi] | (wi < 7 ? (uint64_t)anc[min(wi + 1, 7)] << 32 : 0ull);
  const uint32_t bits = (uint32_t)(win >> (at & 31)) << pre | ((1u << pre) - 1u);
  const int valid = min(max(nkeys - k0, 0), 8);
  return bits & ((1u << valid) - 1u);
}

// Row r of a KV head's group as (token, query head of the group); inv_g = 1 / G.
__device__ __forceinline__ const uint16_t *query_row(const QuantAttnArgs &a, int g, int G, float inv_g,
                                                     int r, int &t) {
  t = (int)(((float)r + 0.5f) * inv_g);  // r / G for r < 2^20
  return (const uint16_t *)a.q + ((size_t)t * a.n_heads + g * G + (r - t * G)) * a.head_dim;
}

template <int D, int FMT, int RT>
__global__ __launch_bounds__(kT, 2) void k_attn_quant(QuantAttnArgs a, TreeMasks tree) {
  typedef Tiles<D, FMT, RT, RT == 3> T;
  constexpr int KSD = T::KSD, NF = T::NF;
  constexpr int RB = 16 * RT;
  constexpr int HD = D / 2;  // dimensions the waves' sums meet in at a time
  constexpr int SOW = kNW * RB * (HD + 4), MW = 2 * SB_MAX_ROWS * 8;
  __shared__ __attribute__((aligned(16))) uint16_t sq[RB][D + 8];  // queries: binary16, scaled
  __shared__ __attribute__((aligned(16))) uint16_t sb[RB][D + 8];  // bfloat16
  __shared__ float sqs[RB];                                         // score multiplier of a row
  __shared__ float sm[kNW][RB], sl[kNW][RB];
  // the ancestor masks during the steps, the waves' sums after them
  __shared__ __attribute__((aligned(16))) float area[SOW > MW ? SOW : MW];
  uint32_t(*sanc)[8] = (uint32_t(*)[8])area;
  float(*so)[RB][HD + 4] = (float(*)[RB][HD + 4]) area;

  const int w = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int lane = threadIdx.x & 63;
  const int lr = lane & 15, lg = lane >> 4;
  const int G = a.n_heads / a.n_kv, R = a.n_tok * G;
  const Range rg = range_of(a);
  if (!rg.live) return;
  const float c = a.scale * 1.44269504088896340736f;  // exp(x scale) = exp2(x c)
  const float inv_g = 1.0f / (float)G;

  // ---- every load before anything waits: the query rows, whose wait then covers
  // only them (loads complete in order), the scales, the wave's first block
  constexpr int TPR = D / 8;  // threads per row
  constexpr int QPT = (RB * TPR + kT - 1) / kT;
  uint4 xq[QPT];
#pragma unroll
  for (int j = 0; j < QPT; ++j) {
    const int i = threadIdx.x + j * kT, r = rg.rb * RB + i / TPR;
    int t;
    xq[j] = make_uint4(0, 0, 0, 0);
    if (i < RB * TPR && r < R)
      xq[j] = *(const uint4 *)(query_row(a, rg.g, G, inv_g, r, t) + (i % TPR) * 8);
  }
  // The wave's steps of the range are w, w + kNW, ...: the tail's, whose 2 NF
  // fragments take the registers of a block's, then blocks.  Blocks and keys past
  // the last read zeros.
  const int bytes = a.cap_blocks * SB_KV_BLOCK * D;  // one head's codes: at most 2^27
  const int nkeys = a.tail_len + a.n_tok, tbytes = a.tail_cap * D * 2;
  const __amdgpu_buffer_rsrc_t krs = uniform_rsrc(a.k8 + (size_t)rg.g * bytes, bytes);
  const __amdgpu_buffer_rsrc_t vrs = uniform_rsrc(a.v8 + (size_t)rg.g * bytes, bytes);
  const __amdgpu_buffer_rsrc_t tks = uniform_rsrc(a.tk + (size_t)rg.g * a.tail_cap * D, tbytes);
  const __amdgpu_buffer_rsrc_t tvs = uniform_rsrc(a.tv + (size_t)rg.g * a.tail_cap * D, tbytes);
  const int nt = rg.t1 - rg.t0, nu = nt + rg.b1 - rg.b0;
  i32x4 kf[NF], vf[NF];
  auto load_block = [&](i32x4 (&f)[NF], __amdgpu_buffer_rsrc_t rs, int u) {
    const int vo = u < nu ? (rg.b0 + u - nt) * (SB_KV_BLOCK * D) + lane * 16 : bytes;
#pragma unroll
    for (int i = 0; i < NF; ++i) f[i] = __builtin_amdgcn_raw_buffer_load_b128(rs, vo, i * 1024, 0);
  };
  auto load_k = [&](int u) {
    if (u >= nt) {
      if (u < nu) load_block(kf, krs, u);
      return;
    }
    // row rho of key tile i is key 8 (rho / 4) + 4 i + rho % 4
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      const int slot = (rg.t0 + u) * 32 + 8 * (lr >> 2) + 4 * i + (lr & 3);
      const int vo = slot < nkeys ? (slot * D + 8 * lg) * 2 : tbytes;
#pragma unroll
      for (int j = 0; j < KSD; ++j)
        kf[i * KSD + j] = __builtin_amdgcn_raw_buffer_load_b128(tks, vo, j * 64, 0);
    }
  };
  auto load_tail_v = [&](int u, int dt) {
    const int key = (rg.t0 + u) * 32 + 8 * lg;
    return __builtin_amdgcn_raw_buffer_load_b128(
        tvs, key < nkeys ? ((16 * dt + lr) * a.tail_cap + key) * 2 : tbytes, 0, 0);
  };
  auto load_v = [&](int u) {
    if (u >= nt) {
      if (u < nu) load_block(vf, vrs, u);
      return;
    }
#pragma unroll
    for (int i = 0; i < NF; ++i) vf[i] = load_tail_v(u, i);
  };
  // the wave's first block, and the blocks' scales
  const int first = rg.b0 + (w < nt ? (w - nt) & (kNW - 1) : w - nt);
  Scales sc{0.0f, 0.0f};
  sc.load(a, rg.g, first, kNW, rg.b1);
  load_k(w);
  load_v(w);
  __builtin_amdgcn_sched_barrier(0);

  // ---- the rows' queries into LDS
#pragma unroll
  for (int j = 0; j < QPT; ++j) {
    const int i = threadIdx.x + j * kT, rr = i / TPR, d0 = (i % TPR) * 8;
    if (i >= RB * TPR) break;  // whole waves
    *(uint4 *)&sb[rr][d0] = xq[j];
    uint32_t top = largest_bits(xq[j]);
#pragma unroll
    for (int o = TPR / 2; o > 0; o >>= 1) top = max(top, (uint32_t)__shfl_xor((int)top, o, 64));
    float mult;
    *(uint4 *)&sq[rr][d0] = scale_query(xq[j], top, c, mult);
    if (d0 == 0) sqs[rr] = mult;
  }
  if (nt) stage_masks(a, tree, (uint4(*)[2])sanc, (uint4(*)[2])(sanc + SB_MAX_ROWS));
  __syncthreads();

  T tl;
  tl.init();
  int u = w;
  float unscale = 1.0f;  // of the output sums
  auto seen = [&](int rt, int k0) {
    const int r = rg.rb * RB + rt * 16 + lr;
    return tail_visible(sanc[r < R ? (int)(((float)r + 0.5f) * inv_g) : 0], k0, a.tail_len, nkeys);
  };
  // A tree row's V that is not finite must not reach the rows that do not see it, as 0
  // times it is NaN: it is taken out of the products and shown afterwards.
  bool bad = false;
  for (; u < nt; u += kNW) {
    const int k0 = (rg.t0 + u) * 32 + 8 * lg;  // this lane's 8 keys
    const bool all = (rg.t0 + u + 1) * 32 <= a.tail_len;
    if ((rg.t0 + u + 1) * 32 > nkeys) {  // slots never written count as zero in V too (0 x NaN)
      const int valid = nkeys - k0;
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        const int keep = (int)((2 * e < valid ? 0x0000ffffu : 0u) | (2 * e + 1 < valid ? 0xffff0000u : 0u));
#pragma unroll
        for (int dt = 0; dt < NF; ++dt) vf[dt][e] &= keep;
      }
    }
    if (!all) bad |= take_not_finite(vf);
    tl.tail([&](int rt, int j) { return as_bf16x8(*(const uint4 *)&sb[rt * 16 + lr][32 * j + 8 * lg]); },
            [&](int i, int j) { return __builtin_bit_cast(bf16x8, kf[i * KSD + j]); },
            [&](int dt) { return __builtin_bit_cast(bf16x8, vf[dt]); },
            [&](int rt) { return all ? 0xffu : seen(rt, k0); }, c, [&]() { load_k(u + kNW); });
    load_v(u + kNW);
  }
  if (bad)
    for (int s = w; s < nt; s += kNW) {
      const int key = (rg.t0 + s) * 32 + 8 * lg;
#pragma unroll
      for (int dt = 0; dt < NF; ++dt)
        tl.show_not_finite(dt, load_tail_v(s, dt), [&](int rt) { return seen(rt, key); });
    }
  if (u < nu) {
    float vtop = sc.largest_v(a, rg.g, first, kNW, rg.b1);
    if (nt) {
      // the tail's sums go on in the blocks' units, within float32: the unit is
      // no smaller than 2^-60 of them
      vtop = fmaxf(vtop, tl.largest_out() * 0x1p-60f);
      tl.scale_out(0x1p15f / vtop);
    }
    unscale = vtop * 0x1p-15f;
    const float rv = 0x1p15f / vtop;
    int at = 0;  // lane that holds the block's scales
    for (; u < nu; u += kNW) {
      // the query fragments are read again for every block: in registers over the
      // loop they would push others into memory
      asm volatile("" ::: "memory");
      if (at == 64) {
        sc.load(a, rg.g, rg.b0 + u - nt, kNW, rg.b1);
        at = 0;
      }
      const BlockScale bs(sc, at++, rv);
      tl.block(
          [&](int rt, int j) {
            return __builtin_bit_cast(f16x8, *(const uint4 *)&sq[rt * 16 + lr][32 * j + 8 * lg]);
          },
          [&](int i, int h) { return make_uint2((uint32_t)kf[i][2 * h], (uint32_t)kf[i][2 * h + 1]); },
          [&](int i, int h) { return make_uint2((uint32_t)vf[i][2 * h], (uint32_t)vf[i][2 * h + 1]); },
          [&](int rt) { return sqs[rt * 16 + lr]; }, bs, [&]() { load_block(kf, krs, u + kNW); });
      load_block(vf, vrs, u + kNW);
    }
  }

  // ---- the waves' sums, in wave order, against the largest maximum; HD
  // dimensions at a time
#pragma unroll
  for (int rt = 0; rt < RT; ++rt) {
    const float sum = sum_x32(sum_x16(tl.l[rt]));
    if (lg == 0) {
      sm[w][rt * 16 + lr] = tl.m[rt];
      sl[w][rt * 16 + lr] = sum;
    }
  }
  __syncthreads();
#pragma unroll
  for (int rt = 0; rt < RT; ++rt) {
    float M = sm[0][rt * 16 + lr];
#pragma unroll
    for (int v = 1; v < kNW; ++v) M = fmaxf(M, sm[v][rt * 16 + lr]);
    const float f = tl.m[rt] == -INFINITY ? 0.0f : __builtin_amdgcn_exp2f(tl.m[rt] - M) * unscale;
#pragma unroll
    for (int dt = 0; dt < NF; ++dt) tl.o[rt][dt] *= f;
  }
  const size_t base = ((size_t)rg.g * a.n_chunks + rg.split) * R;
#pragma unroll
  for (int half = 0; half < 2; ++half) {
    if (half) __syncthreads();
#pragma unroll
    for (int rt = 0; rt < RT; ++rt)
#pragma unroll
      for (int dt = 0; dt < NF / 2; ++dt)
        *(f32x4 *)&so[w][rt * 16 + lr][16 * dt + 4 * lg] = tl.o[rt][half * (NF / 2) + dt];
    __syncthreads();
    for (int i = threadIdx.x; i < RB * (HD / 4); i += kT) {
      const int rr = i / (HD / 4), d0 = (i % (HD / 4)) * 4, r = rg.rb * RB + rr;
      f32x4 x = *(const f32x4 *)&so[0][rr][d0];
#pragma unroll
      for (int v = 1; v < kNW; ++v) x += *(const f32x4 *)&so[v][rr][d0];
      if (r < R) *(f32x4 *)&a.part_o[(base + r) * D + half * HD + d0] = x;
    }
  }
  if (threadIdx.x < RB) {
    const int rr = threadIdx.x, r = rg.rb * RB + rr;
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
hipError_t launch_df(const QuantAttnArgs &a, const TreeMasks &tree, int rt, hipStream_t s) {
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

// Row tiles of a wave and key ranges (attention and merge, us, by the row tiles of a
// KV head):
//  - up to three tiles (six at head_dim 64) one each, so that the waves start and
//    end sooner: 13B, 33 rows, prefix 4096 20.7 against 21.6 with two a wave and
//    29.4 with three; 68M, 65 rows 9.2 against 10.4 and 12.5;
//  - more, two, which halves the codes' conversions: 13B, 65 rows 26.9 against 27.8
//    with one; 13B, 129 rows 37.1 against 43.9 (70B, 33 rows 23.7 against 22.5);
//  - three where the prefix is long and they waste no more of a row block: prefix
//    8192, 13B, 129 rows 57.7 (int8 61.0) against 61.9 (67.6) with two; 70B, 129
//    rows 85.5 against 105.5 (70B, 33 rows, where they leave a quarter of the compute
//    units' places empty, 35.4 against 28.0; 7B, 129 rows 51.0 against 47.9);
//  - two workgroups per compute unit, one where that takes more than eight ranges
//    of a KV head (70B, 5 rows: 10 ranges 13.3, 16 14.2): what a range writes
//    for the merge grows with them.
QuantAttnPlan quant_attn_plan(int n_kv, int head_dim, int n_blocks, int tail_keys, int rows) {
  QuantAttnPlan p{};
  const int tiles = ceil_div(rows, 16), steps = n_blocks + ceil_div(tail_keys, 32);
  if (tiles * head_dim <= 3 * 128)
    p.rt = 1;
  else if (steps >= 128 && ceil_div(tiles, 3) * 3 <= ceil_div(tiles, 2) * 2)
    p.rt = 3;
  else
    p.rt = 2;
  p.n_rb = ceil_div(tiles, p.rt);
  const int groups = n_kv * p.n_rb;
  p.chunks = 2 * kAttnCUs / groups;
  if (p.chunks > 8) p.chunks = 8;
  if (p.chunks * groups < kAttnCUs) p.chunks = kAttnCUs / groups;
  if (p.chunks > kQuantMaxRanges) p.chunks = kQuantMaxRanges;
  if (p.chunks > ceil_div(steps, kNW)) p.chunks = ceil_div(steps, kNW);
  if (p.chunks < 1) p.chunks = 1;
  return p;
}

hipError_t launch_attn_quant(const QuantAttnArgs &args, const TreeArg &tree, hipStream_t s) {
  QuantAttnArgs a = args;
  const QuantAttnPlan p =
      quant_attn_plan(a.n_kv, a.head_dim, a.n_blocks, a.tail_len + a.n_tok, a.n_tok * (a.n_heads / a.n_kv));
  if (a.n_chunks != p.chunks || a.n_tok < 1) return hipErrorInvalidValue;
  a.n_rb = p.n_rb;
  TreeMasks m{};
  if (!a.meta) {  // a parent's row comes before its children's
    for (int i = 0; i < tree.n; ++i) {
      m.parent[i] = tree.parent[i];
      if (tree.n > kMaskArgRows) continue;
      for (int k = 0; k < 4; ++k)
        m.mask[i][k] = (i > 0 ? m.mask[tree.parent[i]][k] : 0u) | ((i >> 5) == k ? 1u << (i & 31) : 0u);
    }
  }
  if (a.head_dim == 128)
    return a.format == SB_KV_INT8 ? launch_df<128, SB_KV_INT8>(a, m, p.rt, s)
                                  : launch_df<128, SB_KV_E4M3>(a, m, p.rt, s);
  if (a.head_dim == 64)
    return a.format == SB_KV_INT8 ? launch_df<64, SB_KV_INT8>(a, m, p.rt, s)
                                  : launch_df<64, SB_KV_E4M3>(a, m, p.rt, s);
  return hipErrorInvalidValue;
}

}  // namespace sb
