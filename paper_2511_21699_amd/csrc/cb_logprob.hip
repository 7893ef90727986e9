// Log probabilities of given tokens, entropies and likeliest tokens of logits rows.  gfx950 only.
//
// With m = max x, Z = sum exp(x - m): log p_t = x_t - m - log Z, entropy = log Z + sum exp(x - m) (m - x) / Z.  Entries of -inf add nothing.
// The likeliest tokens are ordered by one 64-bit word per entry that grows with the value and, among equal values, with falling index
// (amax_word).
#include "cb_logits.h"

namespace cb {

constexpr int kLogprobThreads = 256;

__device__ __forceinline__ float logit_at(const LogprobArgs& a, int64_t row, int i) {
  if (a.is_f32) return as_global((const float*)a.logits)[row * a.stride + i];
  return __uint_as_float((uint32_t)as_global((const uint16_t*)a.logits)[row * a.stride + i] << 16);
}
__device__ __forceinline__ float amax_word_value(unsigned long long w) {
  const uint32_t key = (uint32_t)(w >> 32);
  return __uint_as_float(key & 0x80000000u ? key ^ 0x80000000u : ~key);
}

template <typename X, typename Op>
__device__ __forceinline__ X block_all(X x, X* sh, Op op) {
#pragma unroll
  for (int i = 1; i < 64; i *= 2) {
    if constexpr (sizeof(X) == 8) x = op(x, (X)shfl_u64(x, (threadIdx.x & 63) ^ i));
    else x = op(x, __shfl_xor(x, i, 64));
  }
  __syncthreads();
  if ((threadIdx.x & 63) == 0) sh[threadIdx.x >> 6] = x;
  __syncthreads();
  x = sh[0];
  for (int i = 1; i < kLogprobThreads / 64; i++) x = op(x, sh[i]);
  return x;
}

__global__ __launch_bounds__(kLogprobThreads) void k_logprob(LogprobArgs a) {
  __shared__ float shf[4];
  __shared__ unsigned long long shw[4];
  const int i = blockIdx.x, tid = threadIdx.x;
  const int row = a.rows ? as_global(a.rows)[i] : i;
  const float nan = __uint_as_float(0x7fc00000u);
  if (row < 0 || row >= a.num_rows) {
    if (tid == 0 && a.tokens) as_global(a.logprob)[i] = nan;
    if (tid == 0 && a.entropy) as_global(a.entropy)[i] = nan;
    if (tid < a.top_k) {
      as_global(a.top_tokens)[(int64_t)i * a.top_k + tid] = -1;
      as_global(a.top_logprobs)[(int64_t)i * a.top_k + tid] = nan;
    }
    return;
  }
  unsigned long long best = 0;
  for (int j = tid; j < a.V; j += kLogprobThreads) {
    const unsigned long long w = amax_word(logit_at(a, row, j), j);
    best = w > best ? w : best;
  }
  auto larger = [](unsigned long long x, unsigned long long y) { return x > y ? x : y; };
  auto plus = [](float x, float y) { return x + y; };
  best = block_all(best, shw, larger);
  const float m = amax_word_value(best);
  float z = 0.f, t = 0.f;
  for (int j = tid; j < a.V; j += kLogprobThreads) {
    const float x = logit_at(a, row, j);
    const float e = x == -INFINITY ? 0.f : expf(x - m);
    z += e;
    t += x == -INFINITY ? 0.f : e * (m - x);
  }
  z = block_all(z, shf, plus);
  t = block_all(t, shf, plus);
  const float lz = logf(z);
  auto logp = [&](float x) { return x == -INFINITY ? -INFINITY : (x - m) - lz; };
  if (tid == 0) {
    if (a.tokens) {
      const int tok = as_global(a.tokens)[i];
      as_global(a.logprob)[i] = tok >= 0 && tok < a.V ? logp(logit_at(a, row, tok)) : nan;
    }
    if (a.entropy) as_global(a.entropy)[i] = m == -INFINITY ? 0.f : lz + t / z;
  }
  for (int k = 0; k < a.top_k; k++) {
    if (tid == 0) {
      as_global(a.top_tokens)[(int64_t)i * a.top_k + k] = amax_word_index(best);
      as_global(a.top_logprobs)[(int64_t)i * a.top_k + k] = logp(amax_word_value(best));
    }
    if (k + 1 == a.top_k) break;
    unsigned long long next = 0;
    for (int j = tid; j < a.V; j += kLogprobThreads) {
      const unsigned long long w = amax_word(logit_at(a, row, j), j);
      next = w < best && w > next ? w : next;
    }
    best = block_all(next, shw, larger);
  }
}

hipError_t launch_logprob(hipStream_t st, const LogprobArgs& a) {
  hipLaunchKernelGGL(k_logprob, dim3(a.n), dim3(kLogprobThreads), 0, st, a);
  return hipGetLastError();
}

}  // namespace cb
