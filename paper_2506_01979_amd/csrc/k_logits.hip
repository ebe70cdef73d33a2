// Token counts, and the logits of a token tree under penalties, biases and
// masks with the softmax statistics of the result.
//
// What is computed for token v of row i, every operation rounded on its own:
//   c    = output[v] + #{drafts j on the path root .. i, j >= 1, token v};
//   seen = c > 0 or prompt[v] > 0:  l = l > 0 ? l / rep : l * rep;
//   l -= freq * c;  c > 0: l -= pres;  l += bias[v];  not allowed: -inf.
// Counts are whole numbers below 2^24, exact in float32.
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
  for (int i0 = threadIdx.x; i0 < n; i0 += kBatch * kCountT) {
    int t[kBatch];
#pragma unroll
    for (int b = 0; b < kBatch; ++b) t[b] = i0 + b * kCountT < n ? tokens[i0 + b * kCountT] : -1;
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

__device__ __forceinline__ double wave_sum(double v) {
  for (int o = 32; o > 0; o >>= 1) v += __shfl_xor(v, o, 64);
  return v;
}

// Rows x slices of kT E tokens.  VEC: 16-byte accesses (vocab % 4 == 0 and
// every row and array 16-byte aligned), a thread's tokens in fours; otherwise
// one by one along the slice.  The slice's part of the statistics goes to
// part[row][slice] as the LM head's epilogue leaves it (LmPart).
template <int E, bool VEC>
__global__ __launch_bounds__(kT) void k_shape_logits(ShapeArgs a, TreeArg tree) {
  constexpr int kSpan = kT * E;
  __shared__ int16_t s_jump[SB_MAX_ROWS];
  __shared__ uint8_t s_on[SB_MAX_ROWS];
  __shared__ int s_cnt[kSpan];
  __shared__ float s_best[kT / 64];
  __shared__ int s_arg[kT / 64], s_bad[kT / 64];
  __shared__ double s_sum[kT / 64];
  const int row = blockIdx.y, v0 = blockIdx.x * kSpan, tid = threadIdx.x;
  const float *l = a.logits + (size_t)row * a.vocab;
  float *out = a.out + (size_t)row * a.vocab;
  const uint32_t *mask = a.mask ? a.mask + (size_t)row * a.mask_stride : nullptr;
  // token of element e of this thread
  auto token = [&](int e) { return VEC ? v0 + 4 * (tid + kT * (e >> 2)) + (e & 3) : v0 + tid + kT * e; };
  // every load before the first use; tokens past the vocabulary read as zeros
  float x[E], bias[E];
  int c[E], pr[E];
  uint32_t mw[E];
  auto load = [&](const auto *p, auto (&d)[E], bool there) {
    typedef decltype(d[0] + d[0]) T;
    typedef T V4 __attribute__((ext_vector_type(4)));
    if (VEC) {
#pragma unroll
      for (int e = 0; e < E; e += 4) {
        const V4 t = there && token(e) < a.vocab ? *(const V4 *)(p + token(e)) : V4{0, 0, 0, 0};
#pragma unroll
        for (int i = 0; i < 4; ++i) d[e + i] = t[i];
      }
    } else {
#pragma unroll
      for (int e = 0; e < E; ++e) d[e] = there && token(e) < a.vocab ? p[token(e)] : (T)0;
    }
  };
  load(l, x, true);
  load(a.output, c, a.output != nullptr);
  load(a.prompt, pr, a.prompt != nullptr);
  load(a.bias, bias, a.bias != nullptr);
#pragma unroll
  for (int e = 0; e < E; e += VEC ? 4 : 1)
    mw[e] = mask && token(e) < a.vocab ? mask[token(e) >> 5] : ~0u;

  // ---- the row's drafts in this slice.  Round r marks the 2^r-th ancestors of
  // the rows marked so far, then all jumps double.
  int drafts = 0;
  if (a.count_drafts) {
    const int tok = tid >= 1 && tid < tree.n ? a.tokens[tid] : -1;
    int jump = tid < tree.n ? tree.parent[tid] : -1;
    s_jump[tid] = (int16_t)jump;
    s_on[tid] = tid == row;
#pragma unroll
    for (int e = 0; e < E; ++e) s_cnt[tid + kT * e] = 0;
    __syncthreads();
    for (int step = 1; step < tree.n; step <<= 1) {
      const int next = jump >= 0 ? s_jump[jump] : -1;
      if (jump >= 0 && s_on[tid]) s_on[jump] = 1;
      __syncthreads();
      jump = next;
      s_jump[tid] = (int16_t)next;
      __syncthreads();
    }
    const bool mine = s_on[tid] && tok >= v0 && tok < a.vocab && tok - v0 < kSpan;
    if (mine) atomicAdd(&s_cnt[tok - v0], 1);
    drafts = __syncthreads_or(mine);
  }

  // ---- the rules
  float best = -INFINITY;
  int arg = INT_MAX, bad = 0;
#pragma unroll
  for (int e = 0; e < E; ++e) {
    const int v = token(e);
    float y = x[e];
    const int ci = c[e] + (drafts ? s_cnt[v - v0] : 0);
    const float cf = (float)ci;
    if (ci > 0 || pr[e] > 0) y = y > 0.0f ? y / a.repetition : y * a.repetition;
    y = y - a.frequency * cf;
    if (ci > 0) y = y - a.presence;
    if (a.bias) y = y + bias[e];
    if (!((mw[VEC ? e & ~3 : e] >> (v & 31)) & 1u)) y = -INFINITY;
    x[e] = y;
    if (v < a.vocab) {
      if (isnan(y) || y == INFINITY) bad = 1;
      if (y > best || (y == best && v < arg && y > -INFINITY)) {
        best = y;
        arg = v;
      }
    }
  }
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
  const int lane = tid & 63, w = tid >> 6;
  for (int o = 32; o > 0; o >>= 1) {
    const float ob = __shfl_xor(best, o, 64);
    const int oa = __shfl_xor(arg, o, 64);
    if (ob > best || (ob == best && oa < arg)) {
      best = ob;
      arg = oa;
    }
    bad |= __shfl_xor(bad, o, 64);
  }
  if (lane == 0) {
    s_best[w] = best;
    s_arg[w] = arg;
    s_bad[w] = bad;
  }
  __syncthreads();
  best = s_best[0];
  arg = s_arg[0];
  bad = s_bad[0];
#pragma unroll
  for (int k = 1; k < kT / 64; ++k) {
    if (s_best[k] > best || (s_best[k] == best && s_arg[k] < arg)) {
      best = s_best[k];
      arg = s_arg[k];
    }
    bad |= s_bad[k];
  }
  double sum = 0.0;
  if (!a.greedy) {
    const float m = best == -INFINITY ? 0.0f : best * a.inv_t;
#pragma unroll
    for (int e = 0; e < E; ++e) {
      const float z = x[e] * a.inv_t;
      if (token(e) < a.vocab) sum += (double)expf(z - m);
    }
    sum = wave_sum(sum);
    if (lane == 0) s_sum[w] = sum;
    __syncthreads();
    sum = (s_sum[0] + s_sum[1]) + (s_sum[2] + s_sum[3]);
  }
  if (tid == 0)
    a.part[(size_t)row * gridDim.x + blockIdx.x] = LmPart{best, arg, bad ? (double)NAN : sum};
}

// Tokens per thread: 4 while the launch then has at most four workgroups per
// compute unit and the finishing pass's 256 slices hold the vocabulary.
int shape_e(int vocab, int n_rows) {
  const int64_t g4 = (vocab + kT * 4 - 1) / (kT * 4);
  return g4 <= 256 && g4 * n_rows <= 1024 ? 4 : 16;
}

}  // namespace

int shape_groups(int vocab, int n_rows) {
  const int span = kT * shape_e(vocab, n_rows);
  return (vocab + span - 1) / span;
}

hipError_t launch_shape_logits(const ShapeArgs &a, const TreeArg &tree, int n_rows, hipStream_t s) {
  const dim3 grid(shape_groups(a.vocab, n_rows), n_rows);
  const uintptr_t at = (uintptr_t)a.logits | (uintptr_t)a.out | (uintptr_t)a.output |
                       (uintptr_t)a.prompt | (uintptr_t)a.bias;
  const bool vec = a.vocab % 4 == 0 && (at & 15) == 0;
  if (shape_e(a.vocab, n_rows) == 4) {
    if (vec)
      hipLaunchKernelGGL((k_shape_logits<4, true>), grid, dim3(kT), 0, s, a, tree);
    else
      hipLaunchKernelGGL((k_shape_logits<4, false>), grid, dim3(kT), 0, s, a, tree);
  } else {
    if (vec)
      hipLaunchKernelGGL((k_shape_logits<16, true>), grid, dim3(kT), 0, s, a, tree);
    else
      hipLaunchKernelGGL((k_shape_logits<16, false>), grid, dim3(kT), 0, s, a, tree);
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
