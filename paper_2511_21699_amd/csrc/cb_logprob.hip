// Log probabilities of given tokens, entropies and likeliest tokens of logits rows, in one pass over them.  gfx950 only.
//
// With m = max x, Z = sum exp(x - m), T = sum exp(x - m) (m - x): log p_t = x_t - m - log Z and entropy = log Z + T / Z.  Two parts of a row
// with maxima m <= m' are put together as Z' + f Z and T' + f (T + (m' - m) Z), f = exp(m - m'); so every lane keeps (m, Z, T) of its own
// and they meet at the end.  Differences are cut off at 200, where exp is 0 in 32 bits: -inf (a forbidden token) adds nothing.
//
// The likeliest tokens are ordered by one 64-bit word per entry that grows with the value and, among equal values, with falling index
// (amax_word).  A wavefront's bound is the k-th largest of its lanes' maxima, which at least k entries reach and hardly more do
// (of 4096 normal ones 24 reach the 20th, 44 the 32nd); those that reach it go to a list in LDS, which is cut to its k
// largest at the end.  Of entries equal to the bound the first k (rounded up to a stretch of 64 pieces) are enough: so a row of
// equal entries, or one with few allowed tokens, does not fill the list.
//
// A workgroup takes a row, or a part of one where there are few rows; parts meet through the workspace, and the last to arrive puts them
// together.
#include <float.h>

#include <algorithm>

#include "cb_logits.h"

namespace cb {

#define CB_LDS __attribute__((address_space(3)))
constexpr int kLpVecs = 8;                     // 16-byte pieces that a lane has of a block
constexpr int kLpBlock = 64 * kLpVecs;         // pieces of a block
constexpr int kLpList = 704;                   // entries of a wavefront's list: a stretch of 64 pieces that all go there, and some
constexpr float kLpLog2e = 1.4426950408889634f;
constexpr float kLpFar = 200.f;

__device__ __forceinline__ float amax_word_value(unsigned long long w) {
  const uint32_t key = (uint32_t)(w >> 32);
  return __uint_as_float(key & 0x80000000u ? key ^ 0x80000000u : ~key);
}

struct LpSums {
  float m, z, t;
};
__device__ __forceinline__ void lp_raise(LpSums& s, float m) {  // m >= s.m
  const float d = fminf(m - s.m, kLpFar), f = __builtin_amdgcn_exp2f(-d * kLpLog2e);
  s.t = f * fmaf(d, s.z, s.t);
  s.z *= f;
  s.m = m;
}
__device__ __forceinline__ void lp_join(LpSums& s, LpSums o) {
  const float m = fmaxf(s.m, o.m);
  lp_raise(s, m);
  lp_raise(o, m);
  s.z += o.z;
  s.t += o.t;
}

// The k-th largest of the lanes' values (a bisection over the bits of monotonic words); BITS: 16 where the lower half of a value is 0.
template <int BITS>
__device__ __forceinline__ float lane_kth(float x, int k) {
  const uint32_t key = (uint32_t)(amax_word(x, 0) >> 32);
  uint32_t at = 0;
#pragma unroll
  for (int b = 31; b >= 32 - BITS; b--) {
    const uint32_t next = at | (1u << b);
    if (__popcll(__builtin_amdgcn_ballot_w64(key >= next)) >= k) at = next;
  }
  // (of a negative value the words' lower half is all ones)
  if (BITS == 16 && !(at & 0x80000000u)) at |= 0xffffu;
  return amax_word_value((unsigned long long)at << 32);
}

// A wavefront's list, largest first and no longer than k, in its own place: entries below the bound leave, then every one is put where its
// rank (the number of larger ones) says.
__device__ __forceinline__ int lp_cut(CB_LDS unsigned long long* list, int n, float bound, int k) {
  const int lane = threadIdx.x & 63;
  int kept = 0;
  for (int c = 0; c < n; c += 64) {
    const unsigned long long x = c + lane < n ? list[c + lane] : 0;
    const bool keep = c + lane < n && amax_word_value(x) >= bound;
    const unsigned long long mask = __builtin_amdgcn_ballot_w64(keep);
    wave_lds_sync();  // (writes at or in front of what has been read)
    if (keep) list[kept + __builtin_amdgcn_mbcnt_hi((uint32_t)(mask >> 32), __builtin_amdgcn_mbcnt_lo((uint32_t)mask, 0))] = x;
    kept += __popcll(mask);
  }
  wave_lds_sync();
  constexpr int C = (kLpList + 63) / 64;
  unsigned long long x[C];
  int rank[C];
#pragma unroll
  for (int c = 0; c < C; c++) {
    if (c > 0 && 64 * c >= kept) break;  // (uniform)
    x[c] = 64 * c + lane < kept ? list[64 * c + lane] : 0;
    rank[c] = 64 * c + lane < kept ? 0 : k;
    for (int i = 0; i < kept; i++) rank[c] += list[i] > x[c];
  }
  wave_lds_sync();
#pragma unroll
  for (int c = 0; c < C; c++) {
    if (c > 0 && 64 * c >= kept) break;
    if (rank[c] < k) list[rank[c]] = x[c];
  }
  wave_lds_sync();
  return kept < k ? kept : k;
}

// `lists` sorted lists of up to k entries, `step` entries apart, into the k largest at `out`: an entry's rank is its place and the number of larger
// ones in every other list.
template <typename Count>
__device__ __forceinline__ int lp_merge(const CB_LDS unsigned long long* in, int step, int lists, int k, Count count, CB_LDS unsigned long long* out) {
  int total = 0;
  for (int j = 0; j < lists; j++) total += count(j);
  for (int e = threadIdx.x; e < lists * k; e += blockDim.x) {
    const int mine = e / k, at = e - mine * k;
    if (at >= count(mine)) continue;
    const unsigned long long x = in[mine * step + at];
    int rank = at;
    for (int j = 0; j < lists; j++) {
      if (j == mine) continue;
      int lo = 0, hi = count(j);  // the first that is smaller
      while (lo < hi) {
        const int mid = (lo + hi) >> 1;
        if (in[j * step + mid] > x) lo = mid + 1;
        else hi = mid;
      }
      rank += lo;
    }
    if (rank < k) out[rank] = x;
  }
  return total < k ? total : k;
}

template <typename T, int NW>
__global__ __launch_bounds__(64 * NW) void k_logprob(LogprobArgs a) {
  constexpr int VEC = 16 / sizeof(T), BITS = 8 * sizeof(T) < 32 ? 16 : 32;
  using Scan = WaveScan<T, kLpVecs>;
  using u32x4 = typename Scan::u32x4;
  __shared__ unsigned long long lists[NW][kLpList], best[CB_MAX_TOP];
  __shared__ LpSums sums[NW];
  __shared__ int counts[NW], last;
  const int tid = threadIdx.x, lane = tid & 63, w = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int i = blockIdx.x / a.parts, part = blockIdx.x - i * a.parts, k = a.top_k;
  const int row = a.rows ? as_global(a.rows)[i] : i;
  const float nan = __uint_as_float(0x7fc00000u);
  if (row < 0 || row >= a.num_rows) {
    if (part != 0) return;
    if (tid == 0 && a.tokens) as_global(a.logprob)[i] = nan;
    if (tid == 0 && a.entropy) as_global(a.entropy)[i] = nan;
    if (tid < k) {
      as_global(a.top_tokens)[(int64_t)i * k + tid] = -1;
      as_global(a.top_logprobs)[(int64_t)i * k + tid] = nan;
    }
    return;
  }
  const CBL_GLOBAL T* const base = as_global((const T*)a.logits) + row * a.stride;
  const int token = a.tokens ? as_global(a.tokens)[i] : -1;
  const float x_token = token >= 0 && token < a.V ? Scan::to_f32(base[token]) : 0.f;
  // The row as single entries up to the first 16-byte border, whole pieces, and single entries behind the last: one of those to a lane
  // of the first part's first wavefront.
  int head = (VEC - (int)(((uintptr_t)base / sizeof(T)) & (VEC - 1))) & (VEC - 1);
  head = head < a.V ? head : a.V;
  const int nv = (a.V - head) / VEC, tail0 = head + nv * VEC;
  const int single = part != 0 || w != 0 ? -1 : lane < head ? lane : lane - head < a.V - tail0 ? tail0 + lane - head : -1;
  const float x_single = single >= 0 ? Scan::to_f32(base[single]) : -INFINITY;

  const int blocks = (nv + kLpBlock - 1) / kLpBlock, each = (blocks + a.parts - 1) / a.parts;
  const int b0 = part * each, b1 = b0 + each < blocks ? b0 + each : blocks;
  const CBL_GLOBAL u32x4* const vp = (const CBL_GLOBAL u32x4*)(base + head);
  constexpr uint32_t kNone = sizeof(T) == 2 ? 0xff80ff80u : 0xff800000u;  // -inf
  auto load = [&](int b, u32x4 (&u)[kLpVecs]) {
#pragma unroll
    for (int v = 0; v < kLpVecs; v++) {
      const int at = b * kLpBlock + 64 * v + lane;
      u[v] = vp[at < nv ? at : nv - 1];
    }
  };
  CB_LDS unsigned long long* const list = (CB_LDS unsigned long long*)lists[w];
  LpSums s{-FLT_MAX, 0.f, 0.f};
  float top = -INFINITY, bound = -INFINITY;  // the lane's largest entry; the wavefront's bound
  int n = 0, equal = 0;                      // entries of the list; those appended that are equal to the bound
  auto append = [&](bool c, float x, int index) {
    const unsigned long long mask = __builtin_amdgcn_ballot_w64(c);
    if (mask == 0) return;
    if (c) list[n + __builtin_amdgcn_mbcnt_hi((uint32_t)(mask >> 32), __builtin_amdgcn_mbcnt_lo((uint32_t)mask, 0))] = amax_word(x, index);
    n += __popcll(mask);
  };
  auto one = [&](float x, LpSums& to) {
    const float d = fminf(to.m - x, kLpFar), e = __builtin_amdgcn_exp2f(d * -kLpLog2e);
    to.z += e;
    to.t = fmaf(d, e, to.t);
  };
  if (w == 0 && part == 0 && head + a.V - tail0 > 0) {  // (uniform)
    s.m = fmaxf(s.m, x_single);
    if (single >= 0) one(x_single, s);
    top = x_single;
    if (k > 0) append(single >= 0, x_single, single);
  }
  u32x4 u[kLpVecs];
  if (b0 + w < b1) load(b0 + w, u);
  for (int b = b0 + w; b < b1; b += NW) {
    u32x4 un[kLpVecs];
    if (b + NW < b1) load(b + NW, un);
    float vm[kLpVecs];
#pragma unroll
    for (int v = 0; v < kLpVecs; v++) {
      if (b + 1 == blocks) {  // (uniform: the last block, whose pieces may end inside)
        const bool real = b * kLpBlock + 64 * v + lane < nv;
#pragma unroll
        for (int x = 0; x < 4; x++) u[v][x] = real ? u[v][x] : kNone;
      }
      vm[v] = Scan::vec_max(u[v]);
    }
    float bm = vm[0];
#pragma unroll
    for (int v = 1; v < kLpVecs; v++) bm = fmaxf(bm, vm[v]);
    lp_raise(s, fmaxf(s.m, bm));
    LpSums s2{s.m, 0.f, 0.f};  // (two chains of sums)
#pragma unroll
    for (int v = 0; v < kLpVecs; v++)
#pragma unroll
      for (int j = 0; j < VEC; j++) one(Scan::elem(u[v], j), (v & 1) ? s2 : s);
    s.z += s2.z;
    s.t += s2.t;
    if (k > 0) {
      top = fmaxf(top, bm);
      if (__builtin_amdgcn_ballot_w64(bm > bound || (bm == bound && equal < k)) != 0) {
        const float kth = lane_kth<BITS>(top, k);
        if (kth > bound) {
          bound = kth;
          equal = 0;
        }
#pragma unroll
        for (int v = 0; v < kLpVecs; v++) {
          const bool ties = equal < k;  // (uniform)
          if (__builtin_amdgcn_ballot_w64(vm[v] > bound || (vm[v] == bound && ties)) == 0) continue;
          if (n + 64 * VEC > kLpList) n = lp_cut(list, n, bound, k);
          const int at = b * kLpBlock + 64 * v + lane;
          const bool real = at < nv;
#pragma unroll
          for (int j = 0; j < VEC; j++) {
            const float x = Scan::elem(u[v], j);
            const bool same = real && x == bound;
            append((real && x > bound) || (same && ties), x, head + at * VEC + j);
            equal += __popcll(__builtin_amdgcn_ballot_w64(same));
          }
        }
      }
    }
#pragma unroll
    for (int v = 0; v < kLpVecs; v++) u[v] = un[v];
  }
  // lanes, wavefronts
#pragma unroll
  for (int x = 1; x < 64; x *= 2) lp_join(s, LpSums{__shfl_xor(s.m, x, 64), __shfl_xor(s.z, x, 64), __shfl_xor(s.t, x, 64)});
  if (lane == 0) sums[w] = s;
  if (k > 0) {
    wave_lds_sync();
    n = lp_cut(list, n, bound, k);
    if (lane == 0) counts[w] = n;
  }
  __syncthreads();
  CB_LDS unsigned long long* const out = (CB_LDS unsigned long long*)best;
  int found = k > 0 ? lp_merge((const CB_LDS unsigned long long*)lists[0], kLpList, NW, k, [&](int j) { return counts[j]; }, out) : 0;
  s = sums[0];
#pragma unroll
  for (int x = 1; x < NW; x++) lp_join(s, sums[x]);
  __syncthreads();
  if (a.parts > 1) {
    // The part's state, written through to memory; the row's last part to arrive reads all of them past its own caches.
    const int stride = kLpHeader + k;
    CBL_GLOBAL unsigned long long* const parts = as_global(a.partial) + (int64_t)i * a.parts * stride;
    CBL_GLOBAL unsigned long long* const mine = parts + (int64_t)part * stride;
    auto put = [&](int at, unsigned long long x) { __hip_atomic_store(mine + at, x, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT); };
    if (tid < found) put(kLpHeader + tid, out[tid]);
    if (tid == 0) {
      put(0, (unsigned long long)__float_as_uint(s.m) | ((unsigned long long)__float_as_uint(s.z) << 32));
      put(1, (unsigned long long)__float_as_uint(s.t) | ((unsigned long long)(uint32_t)found << 32));
    }
    asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
    __syncthreads();
    if (tid == 0) {
      CBL_GLOBAL uint32_t* const ticket = as_global(a.tickets) + i * kLpTicketStride;
      const uint32_t arrived = __hip_atomic_fetch_add(ticket, 1u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT) + 1;
      last = arrived == (uint32_t)a.parts;
      if (last) __hip_atomic_store(ticket, 0u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);  // ready for the next launch
    }
    __syncthreads();
    if (!last) return;
    auto get = [&](int p, int at) { return __hip_atomic_load(parts + (int64_t)p * stride + at, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT); };
    static_assert(kLpParts * CB_MAX_TOP <= NW * kLpList && kLpParts <= 64, "");
    CB_LDS unsigned long long* const all = (CB_LDS unsigned long long*)lists[0];
    __shared__ int part_counts[kLpParts];
    for (int e = tid; e < a.parts * k; e += 64 * NW) all[e] = get(e / k, kLpHeader + e % k);  // (of a part that found fewer, anything behind its own)
    unsigned long long h0 = 0, h1 = 0;
    if (lane < a.parts) {
      h0 = get(lane, 0);
      h1 = get(lane, 1);
      if (w == 0) part_counts[lane] = (int)(h1 >> 32);
    }
    s = lane < a.parts ? LpSums{__uint_as_float((uint32_t)h0), __uint_as_float((uint32_t)(h0 >> 32)), __uint_as_float((uint32_t)h1)} : LpSums{-FLT_MAX, 0.f, 0.f};
#pragma unroll
    for (int x = 1; x < 64; x *= 2) lp_join(s, LpSums{__shfl_xor(s.m, x, 64), __shfl_xor(s.z, x, 64), __shfl_xor(s.t, x, 64)});
    __syncthreads();
    if (k > 0) found = lp_merge(all, k, a.parts, k, [&](int j) { return part_counts[j]; }, out);
    __syncthreads();
  }
  // (z is 0 where every entry is -inf)
  const float lz = s.z > 0.f ? logf(s.z) : 0.f;
  auto logp = [&](float x) { return x == -INFINITY ? -INFINITY : (x - s.m) - lz; };
  if (tid == 0) {
    if (a.tokens) as_global(a.logprob)[i] = token >= 0 && token < a.V ? logp(x_token) : nan;
    if (a.entropy) as_global(a.entropy)[i] = s.z > 0.f ? lz + s.t / s.z : 0.f;
  }
  if (tid < k) {  // (fewer are found only in a row with NaN)
    const unsigned long long x = tid < found ? out[tid] : amax_word(nan, 0);
    as_global(a.top_tokens)[(int64_t)i * k + tid] = amax_word_index(x);
    as_global(a.top_logprobs)[(int64_t)i * k + tid] = logp(amax_word_value(x));
  }
}

// Parts of a row: where the rows leave compute units idle, so many that a part has 32 KiB.
int logprob_parts(int n, int64_t row_bytes) {
  const int64_t most = std::min<int64_t>(kLpParts, (row_bytes + (32 << 10) - 1) / (32 << 10));
  return (int)std::max<int64_t>(1, std::min<int64_t>(most, kLpWgs / n));
}

hipError_t launch_logprob(hipStream_t st, const LogprobArgs& args) {
  constexpr int NW = 8;
  LogprobArgs a = args;
  a.parts = logprob_parts(a.n, (int64_t)a.V * (a.is_f32 ? 4 : 2));
  if ((int64_t)a.n * a.parts > INT32_MAX) return hipErrorInvalidValue;
  const dim3 grid(a.n * a.parts), block(64 * NW);
  if (a.is_f32) hipLaunchKernelGGL((k_logprob<float, NW>), grid, block, 0, st, a);
  else hipLaunchKernelGGL((k_logprob<uint16_t, NW>), grid, block, 0, st, a);
  return hipGetLastError();
}

}  // namespace cb
