// Log probabilities of given tokens, entropies and likeliest tokens of logits rows, in one pass over them.  gfx950 only.
//
// With m = max x, Z = sum exp(x - m), T = sum exp(x - m) (m - x): log p_t = x_t - m - log Z and entropy = log Z + T / Z.  Two parts of a row
// with maxima m <= m' are put together as Z' + f Z and T' + f (T + (m' - m) Z), f = exp(m - m'); so every lane keeps (m, Z, T) of its own
// and they meet at the end.  Differences are cut off at 200, where exp is 0 in 32 bits: -inf (a forbidden token) adds nothing.
//
// The likeliest tokens are ordered by one 64-bit word per entry that grows with the value and, among equal values, with falling index
// (amax_word).  A wavefront's bound is the k-th largest of its lanes' maxima, which at least k entries reach and hardly more do
// (of 4096 normal ones 24 reach the 20th, 44 the 32nd).  16-byte pieces whose largest entry reaches the bound of that moment wait in LDS; when they
// are many, and at the end with the last bound, which is higher, their entries that reach it go to a list, which is cut to its k
// largest.  Of entries equal to the bound the first k (rounded up to a stretch of 64 pieces) are enough: so a row of
// equal entries, or one with few allowed tokens, does not fill the list.
//
// A workgroup takes a row, or a part of one where there are few rows; parts meet through the workspace, and the last to arrive puts them
// together.
//
// What bounds it: many rows memory (2048 of 33333 in fp32, 273 MB, 54 us, 5.0 TB/s), beside two exponentials' worth of arithmetic per entry; few rows
// what follows the sweep, a launch and, with parts, two round trips to memory (one row of 32000 in bf16 8.4 us, 40 of 128256 with the 20 largest 14.7).
#include <float.h>

#include <algorithm>

#include "cb_logits.h"

namespace cb {

#define CB_LDS __attribute__((address_space(3)))
constexpr int kLpVecs = 4;                     // 16-byte pieces that a lane has of a block
constexpr int kLpBlock = 64 * kLpVecs;         // pieces of a block
constexpr int kLpList = 576;                   // entries of a wavefront's list: 64 pieces' that all go there, and 64
constexpr int kLpPieces = 128;                 // pieces that wait for being looked through
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

// The lanes' states as one, in every lane.
__device__ __forceinline__ LpSums lp_lanes(LpSums s) {
  auto sum = [](float x) {
    return __uint_as_float(wave_allreduce_u32(__float_as_uint(x), [](uint32_t p, uint32_t q) { return __float_as_uint(__uint_as_float(p) + __uint_as_float(q)); }));
  };
  lp_raise(s, wave_max_f32(s.m));
  return LpSums{s.m, sum(s.z), sum(s.t)};
}

// The k-th largest of the lanes' values (a bisection over the bits of monotonic words); BITS: 16 where the lower half of a value is 0.
template <int BITS>
__device__ __forceinline__ float lane_kth(float x, int k) {
  const uint32_t key = (uint32_t)(amax_word(x, 0) >> 32);
  uint32_t at = 0;
#pragma unroll
  for (int b = 30; b >= 32 - BITS; b -= 2) {  // two bits a step
    const int n1 = __popcll(__builtin_amdgcn_ballot_w64(key >= (at | (1u << b)))), n2 = __popcll(__builtin_amdgcn_ballot_w64(key >= (at | (2u << b)))),
              n3 = __popcll(__builtin_amdgcn_ballot_w64(key >= (at | (3u << b))));
    at |= (n3 >= k ? 3u : n2 >= k ? 2u : n1 >= k ? 1u : 0u) << b;
  }
  // (of a negative value the words' lower half is all ones)
  if (BITS == 16 && !(at & 0x80000000u)) at |= 0xffffu;
  return amax_word_value((unsigned long long)at << 32);
}

__device__ __forceinline__ int lanes_below(unsigned long long mask) {
  return __builtin_amdgcn_mbcnt_hi((uint32_t)(mask >> 32), __builtin_amdgcn_mbcnt_lo((uint32_t)mask, 0));
}
// The entries of a list that are not below the bound, to `out` (which may be the list's own beginning); how many.
__device__ __forceinline__ int lp_keep(const CB_LDS unsigned long long* list, int n, float bound, CB_LDS unsigned long long* out) {
  const int lane = threadIdx.x & 63;
  int kept = 0;
  for (int c = 0; c < n; c += 64) {
    const unsigned long long x = c + lane < n ? list[c + lane] : 0;
    const bool keep = c + lane < n && amax_word_value(x) >= bound;
    const unsigned long long mask = __builtin_amdgcn_ballot_w64(keep);
    wave_lds_sync();  // (writes at or in front of what has been read)
    if (keep) out[kept + lanes_below(mask)] = x;
    kept += __popcll(mask);
  }
  wave_lds_sync();
  return kept;
}
// A wavefront puts a list in order, largest first, and cuts it to k: every entry goes where its rank, the number of larger ones, says.  A long list
// loses those below the k-th largest of the lanes' maxima first (87 fp32 rows of 4568, 32 largest: 22.2 us without, 11.5).
__device__ __forceinline__ int lp_sort(CB_LDS unsigned long long* list, int n, int k) {
  const int lane = threadIdx.x & 63;
  if (n > 128) {
    float top = -INFINITY;
    for (int c = lane; c < n; c += 64) top = fmaxf(top, amax_word_value(list[c]));
    n = lp_keep(list, n, lane_kth<32>(top, k), list);
  }
  if (n <= 128) {
    const unsigned long long x0 = lane < n ? list[lane] : 0, x1 = lane + 64 < n ? list[lane + 64] : 0;  // (0 is below every entry)
    int r0 = 0, r1 = 0;
    auto count = [&](unsigned long long from, int n_from) {
      for (int i = 0; i < n_from; i += 8) {
#pragma unroll
        for (int j = 0; j < 8; j++) {
          const unsigned long long y = (unsigned long long)(uint32_t)__builtin_amdgcn_readlane((int)(uint32_t)from, i + j) |
                                       ((unsigned long long)(uint32_t)__builtin_amdgcn_readlane((int)(uint32_t)(from >> 32), i + j) << 32);
          r0 += y > x0;
          r1 += y > x1;
        }
      }
    };
    count(x0, n < 64 ? n : 64);
    if (n > 64) count(x1, n - 64);
    wave_lds_sync();
    if (x0 != 0 && r0 < k) list[r0] = x0;
    if (x1 != 0 && r1 < k) list[r1] = x1;
  } else {
    // (rare) the largest, the next one, ...; lane r keeps the r-th
    unsigned long long mine = 0, last = ~0ull;
    for (int r = 0; r < k; r++) {
      unsigned long long top = 0;
      for (int c = lane; c < n; c += 64) {
        const unsigned long long x = list[c];
        top = x < last && x > top ? x : top;
      }
#pragma unroll
      for (int i = 1; i < 64; i *= 2) {
        const unsigned long long x = shfl_u64(top, lane ^ i);
        top = x > top ? x : top;
      }
      last = top;
      mine = lane == r ? top : mine;
    }
    wave_lds_sync();
    if (lane < k) list[lane] = mine;
  }
  wave_lds_sync();
  return n < k ? n : k;
}

template <typename T, int NW>
__global__ __launch_bounds__(64 * NW) void k_logprob(LogprobArgs a) {
  constexpr int VEC = 16 / sizeof(T), BITS = 8 * sizeof(T) < 32 ? 16 : 32;
  using Scan = WaveScan<T, kLpVecs>;
  using u32x4 = typename Scan::u32x4;
  __shared__ unsigned long long lists[NW][kLpList], best[NW * CB_MAX_TOP];
  __shared__ u32x4 pieces[NW][kLpPieces];
  __shared__ int piece_at[NW][kLpPieces];
  __shared__ LpSums sums[NW];
  __shared__ float2 bounds[NW];
  __shared__ int found_all, last;
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
  int n = 0, waiting = 0;                    // entries of the list; pieces that wait
  int equal = 0;                             // those taken whose largest entry is the bound
  int refresh = 0;                           // blocks until the bound is worked out again, and
  int every = 1;                             // from then to the next time
  auto pick_elem = [&](const u32x4& v, int j) {  // (j differs between lanes)
    const int d = sizeof(T) == 2 ? j >> 1 : j;
    const uint32_t lo = d & 1 ? v[1] : v[0], hi = d & 1 ? v[3] : v[2], x = d & 2 ? hi : lo;
    return __uint_as_float(sizeof(T) == 4 ? x : j & 1 ? x & 0xffff0000u : x << 16);
  };
  auto to_list = [&](bool c, float x, int index) {
    const unsigned long long mask = __builtin_amdgcn_ballot_w64(c);
    if (c) list[n + lanes_below(mask)] = amax_word(x, index);
    n += __popcll(mask);
  };
  // the waiting pieces' entries that are not below `least` to the list
  auto look_through = [&](float least) {
    wave_lds_sync();
    for (int c = 0; c < waiting; c += 64) {
      if (n + 64 * VEC > kLpList) {
        n = lp_keep(list, n, least, list);
        if (n + 64 * VEC > kLpList) n = lp_sort(list, n, k);
      }
      const bool has = c + lane < waiting;
      const u32x4 piece = ((const CB_LDS u32x4*)pieces[w])[has ? c + lane : 0];
      const int at = ((const CB_LDS int*)piece_at[w])[has ? c + lane : 0];
      uint32_t pick = 0;
#pragma unroll
      for (int j = 0; j < VEC; j++) pick |= Scan::elem(piece, j) >= least ? 1u << j : 0u;
      for (pick = has ? pick : 0u; __builtin_amdgcn_ballot_w64(pick != 0) != 0; pick &= pick - 1) {
        const int j = __builtin_ctz(pick | 0x100u);
        to_list(pick != 0, pick_elem(piece, j), head + at * VEC + j);
      }
    }
    wave_lds_sync();
    waiting = 0;
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
    if (k > 0) to_list(single >= 0, x_single, single);
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
      // (unpacked again further down: kept, the entries would take twice the registers)
      asm volatile("" : "+v"(u[v]));
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
#pragma unroll
    for (int v = 0; v < kLpVecs; v++) asm volatile("" : "+v"(u[v]));
    s.z += s2.z;
    s.t += s2.t;
    if (k > 0) {
      top = fmaxf(top, bm);
      if (--refresh < 0) {  // (after the first block, the second, fourth, eighth: a bound that is behind takes twice the pieces at most)
        const float kth = lane_kth<BITS>(top, k);
        if (kth > bound) {
          bound = kth;
          equal = 0;
        }
        refresh = every - 1;
        every *= 2;
      }
      if (__builtin_amdgcn_ballot_w64(bm > bound || (bm == bound && equal < k)) != 0) {
#pragma unroll
        for (int v = 0; v < kLpVecs; v++) {
          const int at = b * kLpBlock + 64 * v + lane;
          const bool same = vm[v] == bound && equal < k, take = (vm[v] > bound || same) && at < nv;
          const unsigned long long mask = __builtin_amdgcn_ballot_w64(take);
          if (mask == 0) continue;
          if (waiting + 64 > kLpPieces) look_through(bound);
          const int to = waiting + lanes_below(mask);
          if (take) {
            ((CB_LDS u32x4*)pieces[w])[to] = u[v];
            ((CB_LDS int*)piece_at[w])[to] = at;
          }
          waiting += __popcll(mask);
          equal += __popcll(__builtin_amdgcn_ballot_w64(same && take));
        }
      }
    }
#pragma unroll
    for (int v = 0; v < kLpVecs; v++) u[v] = un[v];
  }
  // lanes, wavefronts
  s = lp_lanes(s);
  CB_LDS unsigned long long* const out = (CB_LDS unsigned long long*)best;
  if (lane == 0) sums[w] = s;
  if (k > 0) {
    // A bound for the workgroup: the highest of the wavefronts' bounds, or what a k-th part of the entries reaches in every one.
    const float share = lane_kth<BITS>(top, (k + NW - 1) / NW);
    if (lane == 0) bounds[w] = float2{bound, share};
    if (tid == 0) found_all = 0;
    __syncthreads();
    float high = bounds[0].x, low = bounds[0].y;
#pragma unroll
    for (int x = 1; x < NW; x++) {
      high = fmaxf(high, bounds[x].x);
      low = fminf(low, bounds[x].y);
    }
    const float least = fmaxf(high, low);
    look_through(least);
    n = lp_keep(list, n, least, list);
    if (n > CB_MAX_TOP) n = lp_sort(list, n, k);
    int first = 0;
    if (lane == 0) first = __hip_atomic_fetch_add(&found_all, n, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_WORKGROUP);
    first = __builtin_amdgcn_readfirstlane(first);
    if (lane < n) out[first + lane] = list[lane];
    __syncthreads();
    if (w == 0) lp_sort(out, found_all, k);
  }
  __syncthreads();
  int found = k > 0 ? (found_all < k ? found_all : k) : 0;
  s = sums[0];
#pragma unroll
  for (int x = 1; x < NW; x++) lp_join(s, sums[x]);
  if (a.parts > 1) {
    // The part's state, written through to memory; the row's last part to arrive reads all of them past its own caches.
    const int stride = kLpHeader + k;
    CBL_GLOBAL unsigned long long* const parts = as_global(a.partial) + (int64_t)i * a.parts * stride;
    CBL_GLOBAL unsigned long long* const mine = parts + (int64_t)part * stride;
    auto put = [&](int at, unsigned long long x) { __hip_atomic_store(mine + at, x, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT); };
    if (tid < k) put(kLpHeader + tid, tid < found ? out[tid] : 0ull);
    if (tid == 0) {
      put(0, (unsigned long long)__float_as_uint(s.m) | ((unsigned long long)__float_as_uint(s.z) << 32));
      put(1, (unsigned long long)__float_as_uint(s.t));
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
    static_assert(kLpParts * CB_MAX_TOP <= kLpList && kLpParts <= 64, "");
    if (w != 0) return;
    unsigned long long h0 = 0, h1 = 0;
    const bool one_of = lane < a.parts;
    if (one_of) {
      h0 = get(lane, 0);
      h1 = get(lane, 1);
    }
    constexpr int C = kLpParts * CB_MAX_TOP / 64;
    unsigned long long x[C];
#pragma unroll
    for (int c = 0; c < C; c++) {
      const int e = 64 * c + lane;
      x[c] = 0;
      if (64 * c < a.parts * k) x[c] = e < a.parts * k ? get(e / k, kLpHeader + e % k) : 0;
    }
    s = one_of ? LpSums{__uint_as_float((uint32_t)h0), __uint_as_float((uint32_t)(h0 >> 32)), __uint_as_float((uint32_t)h1)} : LpSums{-FLT_MAX, 0.f, 0.f};
    s = lp_lanes(s);
    if (k > 0) {
      // (a bound as for the wavefronts: the highest k-th entry of a part, or what the parts' shares of k reach in every one; places of a part that
      // found fewer hold 0)
      const int share = (k + a.parts - 1) / a.parts;
      const unsigned long long kth = one_of ? get(lane, kLpHeader + k - 1) : 0, sth = one_of ? get(lane, kLpHeader + share - 1) : 0;
      const float high = wave_max_f32(kth ? amax_word_value(kth) : -INFINITY), low = -wave_max_f32(!one_of ? -INFINITY : sth ? -amax_word_value(sth) : INFINITY);
      const float least = fmaxf(high, low);
      int n_all = 0;
#pragma unroll
      for (int c = 0; c < C; c++) {
        if (64 * c >= a.parts * k) break;
        const bool keep = x[c] != 0 && amax_word_value(x[c]) >= least;
        const unsigned long long mask = __builtin_amdgcn_ballot_w64(keep);
        if (keep) list[n_all + lanes_below(mask)] = x[c];
        n_all += __popcll(mask);
      }
      wave_lds_sync();
      found = lp_sort(list, n_all, k);
      if (lane < found) out[lane] = list[lane];
      wave_lds_sync();
    }
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

template <int NW>
hipError_t launch_waves(hipStream_t st, const LogprobArgs& a) {
  const dim3 grid(a.n * a.parts), block(64 * NW);
  if (a.is_f32) hipLaunchKernelGGL((k_logprob<float, NW>), grid, block, 0, st, a);
  else hipLaunchKernelGGL((k_logprob<uint16_t, NW>), grid, block, 0, st, a);
  return hipGetLastError();
}

// Wavefronts of a workgroup and parts of a row.  What follows a wavefront's sweep (its bound, its list, the workgroup's) takes as long as one to
// two blocks, so rows that fill the chip are taken by few wavefronts, and where they do not, a wavefront has a block or two.  In us, with
// 1, 2, 4 and 8 wavefronts: 4096 rows of 1000 bf16 9.7, 14.7, 21.8, 45.5; 2048 of 32000 44.0, 39.8, 44.0, 50.4; 545 of 128256 108.9, 75.8, 53.4, 60.2;
// 256 of 128256 106.4, 65.6, 40.7, 34.9.  One row of 32000 in 2 parts 9.6, in 4 8.3; one of 128256 in 8 12.2, in 16 16.3.
// In parts, with 4 and 8 wavefronts: 16 rows of 128256 in 8 14.0, 18.6; 60 in 4 18.1, 17.4; 100 in 2 25.3, 20.9; 14 rows of 5000 (one part; with 2 8.3) 7.5, 7.6.
hipError_t launch_logprob(hipStream_t st, const LogprobArgs& args) {
  LogprobArgs a = args;
  const int64_t blocks = ((int64_t)a.V * (a.is_f32 ? 4 : 2) + kLpBlock * 16 - 1) / (kLpBlock * 16);
  a.parts = a.n > kLpWgs / 2 ? 1 : (int)std::max<int64_t>(1, std::min<int64_t>({kLpParts, kLpWgs / a.n, blocks / 4}));
  if (blocks <= 2) return launch_waves<1>(st, a);
  if (a.n >= 1024 || (blocks <= 4 && a.n >= 384)) return launch_waves<2>(st, a);
  if (a.n >= 384 || blocks <= 4 || (a.parts > 2 && blocks < 12 * a.parts)) return launch_waves<4>(st, a);
  return launch_waves<8>(st, a);
}

}  // namespace cb
