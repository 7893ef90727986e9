// Attention of a chunk of new tokens over the cache, one query row to a wavefront.  gfx950 only.
//
// Token i of a sequence with S cached slots attends to slots 0 .. S + i: o = sum_j p_j v_j / sum_j p_j, p_j = exp(scale q.k_j - m), in one
// pass with the running maximum m; everything in 32 bits.  A wavefront takes 64 keys at a time: a lane scores one, then owns D / 64 dims
// of the sum.  It takes every shape, at the pace of the plain arithmetic and with K and V read once per row: for blocks of a size that is no
// power of two in bf16, whose keys the matrix-core kernels' loads could not place with shifts, and to compare with.  2048 tokens of 32/32
// heads of 128 behind nothing, in blocks of 24, take 2.8 ms; on the matrix cores, in blocks of 32, 52 us.
#include "cb_internal.h"

namespace cb {

typedef __attribute__((__vector_size__(4 * sizeof(unsigned)))) unsigned u32x4;

constexpr int kRowsWaves = 4;

__device__ __forceinline__ float row_elem(const CBL_GLOBAL float* p) { return *p; }
__device__ __forceinline__ float row_elem(const CBL_GLOBAL uint16_t* p) { return __uint_as_float((uint32_t)*p << 16); }
__device__ __forceinline__ void put_elem(CBL_GLOBAL float* p, float x) { *p = x; }
__device__ __forceinline__ void put_elem(CBL_GLOBAL uint16_t* p, float x) { *p = __builtin_bit_cast(uint16_t, (__bf16)x); }

template <typename T, int D>
__global__ __launch_bounds__(64 * kRowsWaves) void k_chunk_rows(ChunkArgs a, SeqMeta meta) {
  constexpr int E = 16 / sizeof(T), DL = D / 64;
  __shared__ float qs[kRowsWaves][D], ps[kRowsWaves][64];
  __shared__ int64_t at[kRowsWaves][64];
  const SeqMetaLanes ml = seq_meta_prefetch(meta);
  const int w = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), l = threadIdx.x & 63;
  const int64_t row = (int64_t)blockIdx.x * kRowsWaves + w;
  if (row >= (int64_t)a.total * a.Hq) return;  // (no workgroup barrier below)
  const int tok = (int)(row / a.Hq), head = (int)(row - (int64_t)tok * a.Hq) / (a.Hq / a.Hkv);
  const int b = __popcll(__builtin_amdgcn_ballot_w64(ml.o1 <= tok));  // (offsets past the batch are INT_MAX)
  const SeqShape s = seq_shape(ml, b);
  const int seen = s.S + (tok - s.off) + 1;
  const CBL_GLOBAL T* const k = as_global((const T*)a.kv.k);
  const CBL_GLOBAL T* const v = as_global((const T*)a.kv.v);
#pragma unroll
  for (int i = 0; i < DL; i++) qs[w][l + 64 * i] = row_elem(as_global((const T*)a.q) + row * D + l + 64 * i) * a.scale;
  float m = -INFINITY, sum = 0.f, o[DL] = {};
  for (int k0 = 0; k0 < seen; k0 += 64) {
    const int n = seen - k0 < 64 ? seen - k0 : 64;
    const int64_t mine = slot_offset(a.kv, b, k0 + (l < n ? l : n - 1), head);
    at[w][l] = mine;
    asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");  // (the wavefront's own LDS; its accesses run in order)
    float x = 0.f;
#pragma unroll 4
    for (int d = 0; d < D; d += E) {
      const u32x4 kk = *(const CBL_GLOBAL u32x4*)(k + mine + d);
#pragma unroll
      for (int e = 0; e < E; e++) {
        const float y = sizeof(T) == 4 ? __uint_as_float(kk[e % 4]) : __uint_as_float(e & 1 ? kk[e / 2] & 0xffff0000u : kk[e / 2] << 16);
        x = fmaf(y, qs[w][d + e], x);
      }
    }
    x = l < n ? x : -INFINITY;
    float mx = x;
#pragma unroll
    for (int i = 1; i < 64; i *= 2) mx = fmaxf(mx, __shfl_xor(mx, i, 64));
    const float mn = fmaxf(m, mx), alpha = m == -INFINITY ? 0.f : expf(m - mn);
    const float p = l < n ? expf(x - mn) : 0.f;
    m = mn;
    sum = sum * alpha + p;
    ps[w][l] = p;
    asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
#pragma unroll
    for (int i = 0; i < DL; i++) o[i] *= alpha;
    for (int j = 0; j < n; j++) {
      const CBL_GLOBAL T* const vr = v + at[w][j] + l;
#pragma unroll
      for (int i = 0; i < DL; i++) o[i] = fmaf(ps[w][j], row_elem(vr + 64 * i), o[i]);
    }
  }
#pragma unroll
  for (int i = 1; i < 64; i *= 2) sum += __shfl_xor(sum, i, 64);
#pragma unroll
  for (int i = 0; i < DL; i++) put_elem(as_global((T*)a.out) + row * D + l + 64 * i, o[i] / sum);
}

hipError_t launch_chunk_rows(hipStream_t st, const ChunkArgs& a, const SeqMeta& meta, int dtype, int D) {
  const int64_t wgs = ((int64_t)a.total * a.Hq + kRowsWaves - 1) / kRowsWaves;
  if (wgs > INT32_MAX) return hipErrorInvalidValue;
  const dim3 grid((uint32_t)wgs), block(64 * kRowsWaves);
  if (dtype == CB_F32 && D == 64) hipLaunchKernelGGL((k_chunk_rows<float, 64>), grid, block, 0, st, a, meta);
  else if (dtype == CB_F32) hipLaunchKernelGGL((k_chunk_rows<float, 128>), grid, block, 0, st, a, meta);
  else if (D == 64) hipLaunchKernelGGL((k_chunk_rows<uint16_t, 64>), grid, block, 0, st, a, meta);
  else hipLaunchKernelGGL((k_chunk_rows<uint16_t, 128>), grid, block, 0, st, a, meta);
  return hipGetLastError();
}

}  // namespace cb
