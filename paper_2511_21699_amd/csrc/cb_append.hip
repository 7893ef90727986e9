// New tokens into the cache: query and key heads normalised and rotated, K/V to the tokens' slots.  gfx950 only.
//
// A head x of D dims becomes y = x / sqrt(mean(x^2) + eps) * w, and then every pair (a, b) of its leading rotary dims
// (a cos - b sin, b cos + a sin) of the token's position times the pair's frequency.  All of it in 32 bits, rounded once at the store;
// the angle is reduced to a turn in 64 bits, because position * frequency in 32 bits is off by a thousandth of a radian at position 30000.
//
// What bounds it: memory, every head once in and once out: 8192 tokens of 32/32 heads of 128 in bf16, 403 MB, 74 us, 5.4 TB/s.  A few tokens take
// 3.6 to 4.8 us: a launch and two round trips to memory one behind the other, the table's entry, the frequencies and a tree's parents first and then, behind
// the barrier, the heads.
#include "cb_internal.h"

namespace cb {

typedef __attribute__((__vector_size__(4 * sizeof(unsigned)))) unsigned u32x4;

template <typename T>
struct Elems {};  // 16 bytes of T <-> floats
template <>
struct Elems<float> {
  static constexpr int N = 4;
  static __device__ __forceinline__ void unpack(const u32x4& v, float (&f)[4]) {
#pragma unroll
    for (int i = 0; i < 4; i++) f[i] = __uint_as_float(v[i]);
  }
  static __device__ __forceinline__ u32x4 pack(const float (&f)[4]) {
    return u32x4{__float_as_uint(f[0]), __float_as_uint(f[1]), __float_as_uint(f[2]), __float_as_uint(f[3])};
  }
};
template <>
struct Elems<__bf16> {
  static constexpr int N = 8;
  static __device__ __forceinline__ void unpack(const u32x4& v, float (&f)[8]) {
#pragma unroll
    for (int i = 0; i < 4; i++) {
      f[2 * i] = __uint_as_float(v[i] << 16);
      f[2 * i + 1] = __uint_as_float(v[i] & 0xffff0000u);
    }
  }
  static __device__ __forceinline__ u32x4 pack(const float (&f)[8]) {
    typedef float float2v __attribute__((ext_vector_type(2)));
    typedef __bf16 bf16x2v __attribute__((ext_vector_type(2)));
    u32x4 v;
#pragma unroll
    for (int i = 0; i < 4; i++) v[i] = __builtin_bit_cast(uint32_t, __builtin_convertvector((float2v){f[2 * i], f[2 * i + 1]}, bf16x2v));
    return v;
  }
};

constexpr int kAppendThreads = 256;

// One workgroup per token: its angles are worked out once, behind a barrier, and then all its heads' loads are under way at once.  A group of D / 2 / N lanes has a head: a lane holds two 16-byte pieces, dims N c .. and those half of the
// rotated dims further (of the leading ones; of the others, pieces N c .. and half of those further), so that a rotation's pairs are a
// lane's own.
template <typename T, int D>
__global__ __launch_bounds__(kAppendThreads) void k_append(AppendArgs a, SeqMeta meta) {
  constexpr int N = Elems<T>::N, LPH = D / 2 / N, HEADS = kAppendThreads / LPH;
  __shared__ float cs[D / 2], sn[D / 2];
  __shared__ int jump[CB_MAX_NODES], dist[CB_MAX_NODES];
  __shared__ int64_t where;  // the token's slot in the cache, in elements; -1: outside the pool
  const SeqMetaLanes ml = seq_meta_prefetch(meta);
  const int tid = threadIdx.x, tok = blockIdx.x;
  const int b = __popcll(__builtin_amdgcn_ballot_w64(ml.o1 <= tok));  // (offsets past the batch are INT_MAX)
  const SeqShape s = seq_shape(ml, b);
  const int i = tok - s.off;
  int position = s.S + i;
  if (a.parent) {  // the node's depth by pointer jumping: after r rounds every node is 2^r ancestors up, or at its root
    int up = tid < s.N ? sanitized_parent(a.parent, s.off, tid, a.status) : -1, d = up >= 0 ? 1 : 0;
    jump[tid] = up;
    dist[tid] = d;
    for (int r = jump_rounds(s.N - 1); r > 0; r--) {
      __syncthreads();
      const int uu = up >= 0 ? jump[up] : -1, dd = up >= 0 ? dist[up] : 0;
      __syncthreads();
      d += dd;
      up = uu;
      jump[tid] = up;
      dist[tid] = d;
    }
    __syncthreads();
    position = s.S + dist[i];
  }
  if (tid < a.rotary / 2) {
    const double turns = (double)position * (double)as_global(a.inv_freq)[tid] * 0.15915494309189535;  // 1 / (2 pi)
    const float half_turns = (float)(2.0 * (turns - rint(turns)));
    cs[tid] = cospif(half_turns);
    sn[tid] = sinpif(half_turns);
  }
  if (tid == 0) {
    const int slot = s.S + i;
    const int blk = a.kv.block_size > 0 ? as_global(a.kv.block_table)[(int64_t)b * a.kv.max_blocks + slot / a.kv.block_size] : 0;
    const bool out = a.kv.block_size > 0 && (blk < 0 || blk >= a.kv.num_blocks);
    where = out ? -1 : slot_offset(a.kv, b, slot, 0);
    if (out) atomicOr(a.status, 64);
  }
  __syncthreads();
  const int c = tid % LPH, half = a.rotary / 2;
  // the lane's two pieces
  const bool turned = N * c < half;
  const int d0 = a.interleaved ? 2 * N * c : turned ? N * c : a.rotary + N * c - half;
  const int d1 = a.interleaved ? d0 + N : turned ? d0 + half : d0 + (D - a.rotary) / 2;
  const int64_t at = where;
  for (int h = tid / LPH; h < a.Hq + 2 * a.Hkv; h += HEADS) {
    const bool is_q = h < a.Hq, is_v = h >= a.Hq + a.Hkv;
    if (is_q ? !a.q : at < 0) continue;  // (uniform in a head's lanes)
    const int hh = is_q ? h : is_v ? h - a.Hq - a.Hkv : h - a.Hq;
    const CBL_GLOBAL T* const src = is_q ? as_global((const T*)a.q) + tok * a.q_stride : is_v ? as_global((const T*)a.v) + tok * a.v_stride : as_global((const T*)a.k) + tok * a.k_stride;
    CBL_GLOBAL T* const dst = is_q ? as_global((T*)a.q_out) + ((int64_t)tok * a.Hq + h) * D
                                   : as_global((T*)(is_v ? a.kv.v : a.kv.k)) + at + hh * a.kv.head_stride;
    u32x4 x0 = *(const CBL_GLOBAL u32x4*)(src + hh * D + d0), x1 = *(const CBL_GLOBAL u32x4*)(src + hh * D + d1);
    if (!is_v) {
      float f0[N], f1[N];
      Elems<T>::unpack(x0, f0);
      Elems<T>::unpack(x1, f1);
      const float* const w = is_q ? a.q_weight : a.k_weight;
      if (w) {
        float sum = 0.f;
#pragma unroll
        for (int e = 0; e < N; e++) sum = fmaf(f0[e], f0[e], fmaf(f1[e], f1[e], sum));
#pragma unroll
        for (int x = 1; x < LPH; x *= 2) sum += __shfl_xor(sum, x, 64);
        const float r = 1.0f / sqrtf(sum * (1.0f / D) + a.eps);
#pragma unroll
        for (int e = 0; e < N; e++) {
          f0[e] *= r * as_global(w)[d0 + e];
          f1[e] *= r * as_global(w)[d1 + e];
        }
      }
      if (a.interleaved) {
#pragma unroll
        for (int e = 0; e < N; e += 2) {
          if (d0 + e < a.rotary) {
            const float co = cs[(d0 + e) / 2], si = sn[(d0 + e) / 2], y = f0[e];
            f0[e] = y * co - f0[e + 1] * si;
            f0[e + 1] = f0[e + 1] * co + y * si;
          }
          if (d1 + e < a.rotary) {
            const float co = cs[(d1 + e) / 2], si = sn[(d1 + e) / 2], y = f1[e];
            f1[e] = y * co - f1[e + 1] * si;
            f1[e + 1] = f1[e + 1] * co + y * si;
          }
        }
      } else if (turned) {
#pragma unroll
        for (int e = 0; e < N; e++) {
          const float co = cs[d0 + e], si = sn[d0 + e], y = f0[e];
          f0[e] = y * co - f1[e] * si;
          f1[e] = f1[e] * co + y * si;
        }
      }
      x0 = Elems<T>::pack(f0);
      x1 = Elems<T>::pack(f1);
    }
    *(CBL_GLOBAL u32x4*)(dst + d0) = x0;
    *(CBL_GLOBAL u32x4*)(dst + d1) = x1;
  }
}

hipError_t launch_append(hipStream_t st, const AppendArgs& a, const SeqMeta& meta, int dtype, int D, int total) {
  const dim3 grid(total), block(kAppendThreads);
  if (dtype == CB_F32 && D == 64) hipLaunchKernelGGL((k_append<float, 64>), grid, block, 0, st, a, meta);
  else if (dtype == CB_F32) hipLaunchKernelGGL((k_append<float, 128>), grid, block, 0, st, a, meta);
  else if (D == 64) hipLaunchKernelGGL((k_append<__bf16, 64>), grid, block, 0, st, a, meta);
  else hipLaunchKernelGGL((k_append<__bf16, 128>), grid, block, 0, st, a, meta);
  return hipGetLastError();
}

}  // namespace cb
