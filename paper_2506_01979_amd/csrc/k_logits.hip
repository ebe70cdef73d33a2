// Token counts, and the logits of a token tree under penalties, biases and
// masks with the softmax statistics of the result.
//
// What is computed for token v of row i, every operation rounded on its own:
//   c    = output[v] + #{drafts j on the path root .. i, j >= 1, token v};
//   seen = c > 0 or prompt[v] > 0:  l = l > 0 ? l / rep : l * rep;
//   l -= freq * c;  c > 0: l -= pres;  l += bias[v];  not allowed: -inf.
// Counts are whole numbers below 2^24, exact in float32.
//
// The counts of some 30000 tokens and fewer are bound by their launch: 33 tokens of
// 32000 2.6 us, 32768 of 128256 4.6 us; longer lists by the slices that each read all
// of them, 2^20 tokens of 128256 86 us.  The rules: at k_shape_logits.
#pragma clang fp contract(off)

#include <limits.h>
#include <math.h>

#include "sb_device.h"
#include "sb_internal.h"

namespace sb {
namespace {

constexpr int kT = 256;
constexpr int kCountT = 1024;
constexpr int kCountSlice = 1024;

// One workgroup per slice of the vocabulary: it reads every token (from the L2
// after the first) and counts those of its slice in LDS, so the counts need
// no atomics in memory and no clearing pass.
__global__ __launch_bounds__(kCountT) void k_count_tokens(int vocab, int n,
                                                          const int32_t *__restrict__ tokens,
                                                          int accumulate,
                                                          int32_t *__restrict__ counts) {
  __shared__ int cnt[kCountSlice];
  const int v0 = blockIdx.x * kCountSlice;
  const int v = v0 + threadIdx.x;
  int old = 0;
  if (accumulate && v < vocab) old = counts[v];
  cnt[threadIdx.x] = 0;
  __syncthreads();
  constexpr int kBatch = 8;
  // unsigned: the last batch of 2^31 - 1 tokens ends past them
  for (unsigned i0 = threadIdx.x; i0 < (unsigned)n; i0 += kBatch * kCountT) {
    int t[kBatch];
#pragma unroll
    for (int b = 0; b < kBatch; ++b)
      t[b] = i0 + b * kCountT < (unsigned)n ? tokens[i0 + b * kCountT] : -1;
#pragma unroll
    for (int b = 0; b < kBatch; ++b) {
      const unsigned at = (unsigned)t[b] - (unsigned)v0;
      if (t[b] >= 0 && at < (unsigned)kCountSlice) atomicAdd(&cnt[at], 1);
    }
  }
  __syncthreads();
  if (v < vocab) counts[v] = old + cnt[threadIdx.x];
}

// The tokens that a walk committed, one thread each.  Additions of whole
// numbers: their order does not matter.
__global__ __launch_bounds__(SB_MAX_ROWS) void k_count_step(int vocab, int n_rows,
                                                            const int32_t *__restrict__ tokens,
                                                            const sb_step_result *__restrict__ res,
                                                            int32_t *__restrict__ counts) {
  const int plen = min(res->path_len, SB_MAX_ROWS);
  const int j = threadIdx.x;
  int tok = -1;
  if (j == 0) {
    tok = res->next_token;
  } else if (j < plen) {
    const int row = res->path[j];
    if (row >= 1 && row < n_rows) tok = tokens[row];
  }
  if (tok >= 0 && tok < vocab) atomicAdd(&counts[tok], 1);
}

// A value of every lane joined over the wave: pairs, quads, half rows and rows of
// 16 by DPP, then the four rows.  Every lane returns the same value.
template <int kCtrl, typename T>
__device__ __forceinline__ T dpp(T v) {
  uint32_t b[sizeof(T) / 4];
  __builtin_memcpy(b, &v, sizeof(T));
#pragma unroll
  for (uint32_t &x : b) x = (uint32_t)__builtin_amdgcn_update_dpp(0, (int)x, kCtrl, 0xf, 0xf, false);
  __builtin_memcpy(&v, b, sizeof(T));
  return v;
}
template <typename T>
__device__ __forceinline__ T read_lane(T v, int l) {
  uint32_t b[sizeof(T) / 4];
  __builtin_memcpy(b, &v, sizeof(T));
#pragma unroll
  for (uint32_t &x : b) x = (uint32_t)__builtin_amdgcn_readlane((int)x, l);
  __builtin_memcpy(&v, b, sizeof(T));
  return v;
}
template <typename T, typename Op>
__device__ __forceinline__ T wave_join(T v, Op op) {
  v = op(v, dpp<0xB1>(v));   // quad_perm [1,0,3,2]
  v = op(v, dpp<0x4E>(v));   // quad_perm [2,3,0,1]
  v = op(v, dpp<0x141>(v));  // row_half_mirror
  v = op(v, dpp<0x140>(v));  // row_mirror
  return op(op(read_lane(v, 0), read_lane(v, 16)), op(read_lane(v, 32), read_lane(v, 48)));
}

// LDS that one wave writes and reads: its operations stay in order.
__device__ __forceinline__ void wave_sync() {
  __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
  __builtin_amdgcn_wave_barrier();
}

// y / d, correctly rounded, for quotients that `plain` says.  r is 1 / d correctly
// rounded, NaN for d outside [2^-20, 2^20]: y r is then within 1.5 ulp of the
// quotient, one exact residual brings it within one, and from there the next gives
// the rounded quotient (Markstein, 1990).  Quotients below 2^-60 or above 2^100 may
// leave inexact residuals; the compiler's division has about twice the instructions.
__device__ __forceinline__ float quotient(float y, float d, float r) {
  const float q0 = y * r;
  const float q1 = fmaf(fmaf(-q0, d, y), r, q0);
  return fmaf(fmaf(-q1, d, y), r, q1);
}
__device__ __forceinline__ bool plain(float y, float r) {
  return __float_as_uint(y * r) - 0x21800000u < 0x71800000u - 0x21800000u;
}

// e^t for t <= 0: 2^p by the hardware, 1 ulp, with p = t log2(e) rounded and what it
// leaves put back.  0 for t below -200 and NaN, which -200 stands for: e^-200 is below
// float32, and no infinity or NaN reaches what is put back.
__device__ __forceinline__ float exp_below(float t) {
  t = fmaxf(t, -200.0f);
  const float p = t * 0x1.715476p+0f;
  const float rest = fmaf(t, 0x1.4ae0cp-26f, fmaf(t, 0x1.715476p+0f, -p));
  const float e = __builtin_amdgcn_exp2f(p);
  return fmaf(e, rest * 0x1.62e43p-1f, e);
}

// The drafts on every row's path (its ancestors and itself, the root aside), as
// bits: of up to 128 rows an argument of the kernel (2 KB of the 4 that arguments
// have), of larger trees left in the workspace by k_tree_paths.
constexpr int kPathArgRows = 128;
struct PathMasks {
  uint64_t on[kPathArgRows][2];
};

// Row i: each round joins the path of the row that the jump leads to, then the
// jumps double.
__global__ __launch_bounds__(SB_MAX_ROWS) void k_tree_paths(TreeArg tree, uint64_t *paths) {
  __shared__ int16_t s_jump[SB_MAX_ROWS];
  __shared__ uint64_t s_on[SB_MAX_ROWS][4];
  const int i = threadIdx.x;
  uint64_t on[4];
  int jump = i < tree.n ? tree.parent[i] : -1;
#pragma unroll
  for (int k = 0; k < 4; ++k) on[k] = i > 0 && i >> 6 == k ? 1ull << (i & 63) : 0;
  for (int step = 1; step < tree.n; step <<= 1) {
#pragma unroll
    for (int k = 0; k < 4; ++k) s_on[i][k] = on[k];
    s_jump[i] = (int16_t)jump;
    __syncthreads();
    if (jump >= 0) {
#pragma unroll
      for (int k = 0; k < 4; ++k) on[k] |= s_on[jump][k];
      jump = s_jump[jump];
    }
    __syncthreads();
  }
  if (i < tree.n) {
#pragma unroll
    for (int k = 0; k < 4; ++k) paths[i * 4 + k] = on[k];
  }
}

// A wave owns a slice of 64 E tokens of a row and shares nothing with others: no
// barriers, and the finishing pass joins the slices.  VEC: 16-byte accesses (vocab %
// 4 == 0 and every row and array 16-byte aligned), a lane's tokens in fours;
// otherwise one by one along the slice.  The slice's part of the statistics goes to
// part[row][slice] as the LM head's epilogue leaves it (LmPart).
//
// Bound by the logits' way in and out and by the vector unit: 37 rows of 128256
// under every rule are 38 MB of them, 8 us at a copy's rate, and some 45 instructions
// per token; 14.4 us and the finishing pass's 3.9.  Tried and not kept: slices of a
// workgroup with barriers between its waves (18.5), 16 tokens a lane (more registers,
// 0.3 to 1.5 us slower), several rows per wave with the counts read once (the same or
// slower), the penalties on a compacted list of seen tokens (the same at 37 rows,
// slower above).
template <int E, bool VEC>
__global__ __launch_bounds__(kT) void k_shape_logits(ShapeArgs a, PathMasks paths) {
  constexpr int kSlice = 64 * E;
  __shared__ int s_cnt[kT / 64][kSlice];
  const int w = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lane = threadIdx.x & 63;
  const int slice = blockIdx.x * (kT / 64) + w, v0 = slice * kSlice, row = blockIdx.y;
  if (slice >= a.groups) return;
  // place in the slice, and token, of element e of this lane
  auto place = [&](int e) { return VEC ? 4 * (lane + 64 * (e >> 2)) + (e & 3) : lane + 64 * e; };
  auto token = [&](int e) { return v0 + place(e); };
  // every load before the first use; tokens past the vocabulary read as zeros and
  // are not allowed, which keeps them out of the statistics
  auto load = [&](const auto *p, auto (&d)[E]) {
    typedef decltype(d[0] + d[0]) T;
    typedef T V4 __attribute__((ext_vector_type(4)));
    if (VEC) {
#pragma unroll
      for (int e = 0; e < E; e += 4) {
        const V4 t = p && token(e) < a.vocab ? *(const V4 *)(p + token(e)) : V4{0, 0, 0, 0};
#pragma unroll
        for (int i = 0; i < 4; ++i) d[e + i] = t[i];
      }
    } else {
#pragma unroll
      for (int e = 0; e < E; ++e) d[e] = p && token(e) < a.vocab ? p[token(e)] : (T)0;
    }
  };
  // the tree's tokens on the row's path: tree row lane + 64 k
  constexpr int kTok = SB_MAX_ROWS / 64;
  int tok[kTok];
  uint64_t on[kTok];
#pragma unroll
  for (int k = 0; k < kTok; ++k) {
    tok[k] = a.count_drafts && lane + 64 * k < a.n_rows ? a.tokens[lane + 64 * k] : -1;
    on[k] = a.count_drafts && 64 * k < a.n_rows ? (a.paths ? a.paths[row * 4 + k] : paths.on[row][k & 1]) : 0;
  }
  float x[E], bias[E];
  int c[E], pr[E];
  uint32_t allowed[VEC ? E / 4 : E];
  load(a.output, c);
  load(a.prompt, pr);
  load(a.logits + (size_t)row * a.vocab, x);
  load(a.bias, bias);
  const uint32_t *mask = a.mask ? a.mask + (size_t)row * a.mask_stride : nullptr;
#pragma unroll
  for (int e = 0; e < E; e += VEC ? 4 : 1)
    allowed[VEC ? e / 4 : e] = token(e) < a.vocab ? (mask ? mask[token(e) >> 5] : ~0u) : 0u;

  // ---- the drafts on the row's path in this slice
  bool drafts = false;
  if (a.count_drafts) {
    bool mine[kTok];
#pragma unroll
    for (int k = 0; k < kTok; ++k) {
      mine[k] = (on[k] >> lane & 1) && tok[k] >= v0 && tok[k] < a.vocab && tok[k] - v0 < kSlice;
      drafts |= mine[k];
    }
    drafts = __any(drafts);
    if (drafts) {
#pragma unroll
      for (int e = 0; e < E; ++e) s_cnt[w][lane + 64 * e] = 0;
      wave_sync();
#pragma unroll
      for (int k = 0; k < kTok; ++k)
        if (mine[k]) atomicAdd(&s_cnt[w][tok[k] - v0], 1);
      wave_sync();
    }
  }

  // ---- the penalties
  if (a.output || a.prompt || drafts) {
    if (drafts) {
#pragma unroll
      for (int e = 0; e < E; ++e) c[e] += s_cnt[w][place(e)];
    }
    if (a.repetition != 1.0f) {
      bool slow = false;
#pragma unroll
      for (int e = 0; e < E; ++e) slow |= (x[e] > 0.0f) & !plain(x[e], a.inv_repetition);
      if (__any(slow)) {
#pragma unroll 1
        for (int e = 0; e < E; ++e) {
          // one element a turn, in place of element 0: this is rare, and unrolled it
          // would be most of the kernel
          if (max(c[0], pr[0]) > 0) x[0] = x[0] > 0.0f ? x[0] / a.repetition : x[0] * a.repetition;
          const float x0 = x[0];
          const int c0 = c[0], p0 = pr[0];
#pragma unroll
          for (int k = 0; k + 1 < E; ++k) {
            x[k] = x[k + 1];
            c[k] = c[k + 1];
            pr[k] = pr[k + 1];
          }
          x[E - 1] = x0;
          c[E - 1] = c0;
          pr[E - 1] = p0;
        }
      } else {
#pragma unroll
        for (int e = 0; e < E; ++e) {
          const float q = quotient(x[e], a.repetition, a.inv_repetition), p = x[e] * a.repetition;
          const float z = x[e] > 0.0f ? q : p;
          x[e] = max(c[e], pr[e]) > 0 ? z : x[e];
        }
      }
    }
#pragma unroll
    for (int e = 0; e < E; ++e) {
      x[e] = x[e] - a.frequency * (float)c[e];
      x[e] = x[e] - (c[e] > 0 ? a.presence : 0.0f);
    }
  }

  // ---- bias and mask
  if (a.bias) {
#pragma unroll
    for (int e = 0; e < E; ++e) x[e] = x[e] + bias[e];
  }
  float best = -INFINITY;
  bool bad = false;
#pragma unroll
  for (int e = 0; e < E; ++e) {
    const uint32_t bit = VEC ? (allowed[e >> 2] >> (token(e & ~3) & 31)) & (1u << (e & 3))
                             : (allowed[e] >> (token(e) & 31)) & 1u;
    x[e] = bit ? x[e] : -INFINITY;
    bad |= !(x[e] < INFINITY);  // NaN or +inf
    best = fmaxf(best, x[e]);
  }
  float *out = a.out + (size_t)row * a.vocab;
  if (VEC) {
#pragma unroll
    for (int e = 0; e < E; e += 4)
      if (token(e) < a.vocab) *(f32x4 *)(out + token(e)) = f32x4{x[e], x[e + 1], x[e + 2], x[e + 3]};
  } else {
#pragma unroll
    for (int e = 0; e < E; ++e)
      if (token(e) < a.vocab) out[token(e)] = x[e];
  }

  // ---- the slice's part of the statistics
  best = wave_join(best, [](float p, float q) { return fmaxf(p, q); });
  int arg = INT_MAX;  // the first token of the maximum
#pragma unroll
  for (int e = E - 1; e >= 0; --e) arg = x[e] == best ? token(e) : arg;
  arg = wave_join(arg, [](int p, int q) { return min(p, q); });
  double sum = 0.0;
  if (!a.greedy) {
    float m = best * a.inv_t;  // past float32 also from a finite best
    if (m == -INFINITY) m = 0.0f;
    bad |= m == INFINITY;  // z - m is of two infinities
#pragma unroll
    for (int e = 0; e < E; ++e) sum += (double)exp_below(x[e] * a.inv_t - m);
    sum = wave_join(sum, [](double p, double q) { return p + q; });
  }
  bad = __any(bad);
  if (lane == 0)
    a.part[(size_t)row * a.groups + slice] =
        LmPart{best, best == -INFINITY ? INT_MAX : arg, bad ? (double)NAN : sum};
}

// Tokens per lane: 4 while the launch then has at most four workgroups per compute
// unit and the slices are at most 512 (1 row of 32000: 5.4 us with 4, 5.9 with 8).
int shape_e(int vocab, int n_rows) {
  const int64_t g4 = (vocab + 255) / 256;
  return g4 <= 512 && g4 * n_rows <= 4096 ? 4 : 8;
}

}  // namespace

int shape_groups(int vocab, int n_rows) {
  const int slice = 64 * shape_e(vocab, n_rows);
  return (vocab + slice - 1) / slice;
}

size_t shape_path_bytes(int n_rows) {
  return n_rows > kPathArgRows ? (size_t)n_rows * 4 * sizeof(uint64_t) : 0;
}

hipError_t launch_shape_logits(const ShapeArgs &args, const TreeArg &tree, hipStream_t s) {
  ShapeArgs a = args;
  const int n = a.n_rows;
  a.groups = shape_groups(a.vocab, n);
  PathMasks paths;
  if (!a.count_drafts || n <= kPathArgRows) {
    a.paths = nullptr;
    for (int i = 0; a.count_drafts && i < n; ++i)  // a parent's row comes before its children's
      for (int k = 0; k < 2; ++k)
        paths.on[i][k] = i > 0 ? paths.on[tree.parent[i]][k] | (i >> 6 == k ? 1ull << (i & 63) : 0) : 0;
  } else {
    hipLaunchKernelGGL(k_tree_paths, dim3(1), dim3(SB_MAX_ROWS), 0, s, tree, a.paths);
  }
  const uintptr_t at = (uintptr_t)a.logits | (uintptr_t)a.out | (uintptr_t)a.output |
                       (uintptr_t)a.prompt | (uintptr_t)a.bias;
  const bool vec = a.vocab % 4 == 0 && (at & 15) == 0;
  const dim3 grid((a.groups + kT / 64 - 1) / (kT / 64), n);
  if (shape_e(a.vocab, n) == 4) {
    if (vec)
      hipLaunchKernelGGL((k_shape_logits<4, true>), grid, dim3(kT), 0, s, a, paths);
    else
      hipLaunchKernelGGL((k_shape_logits<4, false>), grid, dim3(kT), 0, s, a, paths);
  } else {
    if (vec)
      hipLaunchKernelGGL((k_shape_logits<8, true>), grid, dim3(kT), 0, s, a, paths);
    else
      hipLaunchKernelGGL((k_shape_logits<8, false>), grid, dim3(kT), 0, s, a, paths);
  }
  return hipGetLastError();
}

hipError_t launch_count_tokens(int vocab, int n, const int32_t *tokens, int accumulate,
                               int32_t *counts, hipStream_t s) {
  hipLaunchKernelGGL(k_count_tokens, dim3((vocab + kCountSlice - 1) / kCountSlice), dim3(kCountT), 0,
                     s, vocab, n, tokens, accumulate, counts);
  return hipGetLastError();
}

hipError_t launch_count_step(int vocab, int n_rows, const int32_t *tokens,
                             const sb_step_result *res, int32_t *counts, hipStream_t s) {
  hipLaunchKernelGGL(k_count_step, dim3(1), dim3(SB_MAX_ROWS), 0, s, vocab, n_rows, tokens, res,
                     counts);
  return hipGetLastError();
}

}  // namespace sb
