// Attention of a chunk of new tokens over the cache in fp32 (head_dim 64 or 128) on the matrix cores, gfx950 only.
//
// Token i of a sequence with S cached slots attends to slots 0 .. S + i: o = sum_j p_j v_j / sum_j p_j, p_j = exp(scale q.k_j - m), with products and
// sums in plain fp32 (v_mfma_f32_16x16x4_f32) and the accurate expf.  The g query heads of a kv head are g rows to a token.
//
// A workgroup of 8 wavefronts has RT row tiles of 16 rows of a kv head and a split of their keys.  The wavefronts take units of 16 keys in turn
// and share nothing until the end: K and V go straight from memory to the registers that the MFMAs read, and serve RT tiles.  The
// wavefronts' states are combined through LDS, the splits' by the tile's last workgroup.
// What bounds it: prompts the matrix cores, a unit is RT D / 2 MFMAs of 32 cycles with two wavefronts to a SIMD (heads of 128, two row tiles: busy 62%
// of the launch at 2.19 GHz, the wavefronts waiting 62% of theirs; 32/8 heads, 512 tokens behind 4096 in 372 us, 98 TFLOP/s).  Single tokens the loads on their way:
// a compute unit takes 39 bytes a ns.  One token behind 8192 25 us, 16 behind 2000 each 57 us (4.6 TB/s); with a table's entries asked for
// where they are needed, V not ahead and eight splits at a time in the merge these were 40 and 78.
//
// Register layouts (lane l, r = l % 16, h = l / 16):
//   scores transposed, S^T = K Q^T: MFMA (j, e) contracts the dims 16j + 4h + e; A = K[key r], B = Q[query r], so both
//   are 16-byte pieces of a row, and D[v] = S^T[key 4h+v][query r].
//   O^T = V^T P^T: MFMA (v, n, e) contracts the keys 4h + v; B = the lane's own probability v, A = V[key 4h+v][dim
//   64n + 4r + e], again 16-byte pieces; D[i] = O^T[dim 64n + 16h + 4i + e][query r].
#include <type_traits>

#include "cb_chunk.h"

namespace cb {

typedef __attribute__((__vector_size__(4 * sizeof(float)))) float f32x4;

constexpr int kF32Unit = 16;   // keys per unit
constexpr int kF32Waves = 8;

template <int D, int RT>
struct ChunkF32Lds {
  static constexpr int kStride = D + 4;   // (rows 16 bytes apart in the banks)
  float o[kF32Waves][16 * RT * kStride];
  float2 ml[kF32Waves][16 * RT];
  int last;
};

// Partial states are written through to memory and read past the reader's own L2; two floats at a time.
__device__ __forceinline__ void put_pair(float* p, float a, float b) {
  const unsigned long long x = (unsigned long long)__float_as_uint(a) | ((unsigned long long)__float_as_uint(b) << 32);
  __hip_atomic_store((CBL_GLOBAL unsigned long long*)p, x, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
}
__device__ __forceinline__ float2 get_pair(const float* p) {
  const unsigned long long x = __hip_atomic_load((const CBL_GLOBAL unsigned long long*)p, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
  return float2{__uint_as_float((uint32_t)x), __uint_as_float((uint32_t)(x >> 32))};
}
__device__ __forceinline__ float quarter_max(float x) {  // over the four lanes with equal r
  const auto a = __builtin_amdgcn_permlane16_swap(__float_as_uint(x), __float_as_uint(x), false, false);
  x = fmaxf(__uint_as_float(a[0]), __uint_as_float(a[1]));
  const auto b = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
  return fmaxf(__uint_as_float(b[0]), __uint_as_float(b[1]));
}
__device__ __forceinline__ float state_weight(float m, float ref) { return m == -INFINITY ? 0.f : expf(m - ref); }
__device__ __forceinline__ bool is_finite(float x) { return (__float_as_uint(x) & 0x7f800000u) != 0x7f800000u; }

template <int D, int RT>
__global__ __launch_bounds__(64 * kF32Waves, D == 64 && RT == 1 ? 4 : 2) void k_chunk_f32(AttnParams p, SeqMeta meta, ChunkSplits splits) {
  constexpr int NJ = D / 16, NB = D / 64, ROWS = 16 * RT;
  __shared__ ChunkF32Lds<D, RT> sh;
  const SeqMetaLanes ml = seq_meta_prefetch(meta);
  const int lane_chunk = splits.keys[threadIdx.x & 63];
  const int tid = threadIdx.x, w = __builtin_amdgcn_readfirstlane(tid >> 6), l = tid & 63, r = l & 15, h = l >> 4;
  TileJob jb;
  if (!chunk_job(p, ml, lane_chunk, blockIdx.x, jb)) return;
  const int b = jb.b, hk = jb.hk, k0 = jb.k0, k1 = jb.k1, nsplit = jb.nsplit, nu = (k1 - k0 + kF32Unit - 1) / kF32Unit;
  const int S = jb.S + jb.row0 / jb.g + 1;  // (every row sees the keys below)
  const CBL_GLOBAL float* const kb = (const CBL_GLOBAL float*)p.kv.k;
  const CBL_GLOBAL float* const vb = (const CBL_GLOBAL float*)p.kv.v;
  f32x4 q[RT][NJ];
  int seen[RT];  // keys that the lane's queries see
#pragma unroll
  for (int t = 0; t < RT; t++) {
    int row = jb.row0 + 16 * t + r;
    row = row < jb.M ? row : jb.M - 1;   // (rows past the end repeat the last one and are not written)
    const int token = row / jb.g;
    seen[t] = jb.S + token + 1 < k1 ? jb.S + token + 1 : k1;
    const CBL_GLOBAL f32x4* const qp = (const CBL_GLOBAL f32x4*)((const CBL_GLOBAL float*)p.q + ((int64_t)(jb.off + token) * p.Hq + hk * jb.g + (row - token * jb.g)) * D);
#pragma unroll
    for (int j = 0; j < NJ; j++) q[t][j] = qp[4 * j + h];
  }
  // Where lane l's key of a unit (r) is.  The table's entry is asked for two units ahead and becomes an offset one ahead, so that no load waits for
  // another one's address.  Keys past the split's end repeat its last one (masked below): every address stays inside the sequence.
  auto look_up = [&](int u, int& block, int& slot) {
    int key = k0 + u * kF32Unit + r;
    key = key < k1 ? key : k1 - 1;
    block = b;
    slot = key;
    if (p.kv.block_size > 0) {
      const int lb = key / p.kv.block_size;
      slot = key - lb * p.kv.block_size;
      block = as_global(p.kv.block_table)[(int64_t)b * p.kv.max_blocks + lb];
    }
  };
  auto place = [&](int block, int slot) {
    if (p.kv.block_size > 0) block = block < 0 ? 0 : block >= p.kv.num_blocks ? (int)p.kv.num_blocks - 1 : block;
    return block * p.kv.seq_stride + slot * p.kv.token_stride + hk * p.kv.head_stride;
  };
  auto load_k = [&](int64_t off, f32x4 (&k)[NJ]) {
    const CBL_GLOBAL f32x4* const kp = (const CBL_GLOBAL f32x4*)(kb + off);
#pragma unroll
    for (int j = 0; j < NJ; j++) k[j] = kp[4 * j + h];
  };
  auto load_v = [&](int64_t off, f32x4 (&v)[4][NB]) {
#pragma unroll
    for (int x = 0; x < 4; x++) {
      const uint32_t lo = __builtin_amdgcn_ds_bpermute(4 * (4 * h + x), (int)(uint32_t)off), hi = __builtin_amdgcn_ds_bpermute(4 * (4 * h + x), (int)(off >> 32));
      const CBL_GLOBAL f32x4* const vp = (const CBL_GLOBAL f32x4*)(vb + (int64_t)(((uint64_t)hi << 32) | lo));
#pragma unroll
      for (int n = 0; n < NB; n++) v[x][n] = vp[16 * n + r];
    }
  };
  // K and V are asked for a unit ahead where there are registers for it: V with one row tile, K unless heads of 64 have four wavefronts to a SIMD
  // (then its loads go out when the scores are through with the registers).
  constexpr bool K_AHEAD = RT == 2 || D == 128, V_AHEAD = RT == 1;
  f32x4 k[NJ], v[4][NB];
  int block, slot;
  look_up(w, block, slot);
  int64_t off = place(block, slot);
  load_k(off, k);
  if (V_AHEAD) load_v(off, v);
  look_up(w + kF32Waves, block, slot);
  f32x4 o[RT][NB][4];
  float m[RT], lsum[RT];
#pragma unroll
  for (int t = 0; t < RT; t++) {
#pragma unroll
    for (int n = 0; n < NB; n++)
#pragma unroll
      for (int e = 0; e < 4; e++) o[t][n][e] = f32x4{0.f, 0.f, 0.f, 0.f};
    m[t] = -INFINITY;
    lsum[t] = 0.f;
  }
  for (int u = w; u < nu; u += kF32Waves) {
    f32x4 kn[NJ], vn[4][NB];
    const int64_t next = place(block, slot);
    look_up(u + 2 * kF32Waves, block, slot);
    load_v(V_AHEAD ? next : off, V_AHEAD ? vn : v);
    if (K_AHEAD) load_k(next, kn);
    off = next;
    f32x4 s[RT], s1[RT];
#pragma unroll
    for (int t = 0; t < RT; t++) s[t] = s1[t] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int j = 0; j < NJ; j += 2)
#pragma unroll
      for (int e = 0; e < 4; e++)
#pragma unroll
        for (int t = 0; t < RT; t++) {
          s[t] = __builtin_amdgcn_mfma_f32_16x16x4f32(k[j][e], q[t][j][e], s[t], 0, 0, 0);
          s1[t] = __builtin_amdgcn_mfma_f32_16x16x4f32(k[j + 1][e], q[t][j + 1][e], s1[t], 0, 0, 0);
        }
    if (!K_AHEAD) load_k(next, k);
    const int key0 = k0 + u * kF32Unit;
    const bool masked = key0 + kF32Unit > (S < k1 ? S : k1);  // (uniform)
    bool odd_v = false;
    if (masked) {  // A value that a query must not see reaches its sum with weight 0, which hides it only if it is finite.
      bool bad = false;
#pragma unroll
      for (int x = 0; x < 4; x++)
#pragma unroll
        for (int n = 0; n < NB; n++)
#pragma unroll
          for (int e = 0; e < 4; e++) {
            const bool fin = is_finite(v[x][n][e]);
            bad |= !fin;
            v[x][n][e] = fin ? v[x][n][e] : 0.f;
          }
      odd_v = __builtin_amdgcn_ballot_w64(bad) != 0ull;
    }
    float pr[RT][4];
#pragma unroll
    for (int t = 0; t < RT; t++) {
      f32x4 x = (s[t] + s1[t]) * p.scale;
      if (masked) {
#pragma unroll
        for (int i = 0; i < 4; i++) x[i] = key0 + 4 * h + i < seen[t] ? x[i] : -INFINITY;
      }
      const float mn = fmaxf(m[t], quarter_max(fmaxf(fmaxf(x[0], x[1]), fmaxf(x[2], x[3]))));
      if (__builtin_amdgcn_ballot_w64(mn > m[t]) != 0ull) {
        const float alpha = state_weight(m[t], mn);
#pragma unroll
        for (int n = 0; n < NB; n++)
#pragma unroll
          for (int e = 0; e < 4; e++) o[t][n][e] *= alpha;
        lsum[t] *= alpha;
        m[t] = mn;
      }
#pragma unroll
      for (int i = 0; i < 4; i++) {
        pr[t][i] = state_weight(x[i], m[t]);
        lsum[t] += pr[t][i];
      }
    }
#pragma unroll
    for (int x = 0; x < 4; x++)
#pragma unroll
      for (int n = 0; n < NB; n++)
#pragma unroll
        for (int e = 0; e < 4; e++)
#pragma unroll
          for (int t = 0; t < RT; t++) o[t][n][e] = __builtin_amdgcn_mfma_f32_16x16x4f32(v[x][n][e], pr[t][x], o[t][n][e], 0, 0, 0);
    if (__builtin_expect(odd_v, 0)) {  // infinities or NaN among the unit's values, for the queries that do see them, with a weight of 0 in 32 bits too
#pragma unroll
      for (int x = 0; x < 4; x++)
        for (int part = 0; part < 4 && key0 + 4 * part + x < k1; part++) {
          const CBL_GLOBAL float* const vp = vb + slot_offset(p.kv, b, key0 + 4 * part + x, hk);
#pragma unroll
          for (int t = 0; t < RT; t++) {
            const float pk = __shfl(pr[t][x], 16 * part + r, 64);
#pragma unroll
            for (int n = 0; n < NB; n++)
#pragma unroll
              for (int e = 0; e < 4; e++)
#pragma unroll
                for (int i = 0; i < 4; i++) {
                  const float odd = vp[64 * n + 16 * h + 4 * i + e];
                  o[t][n][e][i] += is_finite(odd) || key0 + 4 * part + x >= seen[t] ? 0.f : (pk == 0.f ? 1.f : pk) * odd;
                }
          }
        }
    }
    if (V_AHEAD) {
#pragma unroll
      for (int x = 0; x < 4; x++)
#pragma unroll
        for (int n = 0; n < NB; n++) v[x][n] = vn[x][n];
    }
    if (K_AHEAD) {
#pragma unroll
      for (int j = 0; j < NJ; j++) k[j] = kn[j];
    }
  }

  // The wavefronts' states into one.  Thread t then owns 4 dims of a row.
  constexpr int PS = partial_stride(D), LS = ChunkF32Lds<D, RT>::kStride;
#pragma unroll
  for (int t = 0; t < RT; t++) {
    lsum[t] += __shfl_xor(lsum[t], 16, 64);
    lsum[t] += __shfl_xor(lsum[t], 32, 64);
#pragma unroll
    for (int n = 0; n < NB; n++)
#pragma unroll
      for (int i = 0; i < 4; i++)
        *reinterpret_cast<f32x4*>(&sh.o[w][(16 * t + r) * LS + 64 * n + 16 * h + 4 * i]) = f32x4{o[t][n][0][i], o[t][n][1][i], o[t][n][2][i], o[t][n][3][i]};
    if (h == 0) sh.ml[w][16 * t + r] = float2{m[t], lsum[t]};
  }
  __syncthreads();
  constexpr int TPR = D / 4, STEP = 64 * kF32Waves / TPR, N = ROWS > STEP ? ROWS / STEP : 1;  // threads of a row, rows at a time, rows of a thread
  const int c = tid % TPR * 4;
  auto row_of = [&](int i) { return tid / TPR + i * STEP; };
  auto live = [&](int i) { return row_of(i) < ROWS && jb.row0 + row_of(i) < jb.M; };
  auto out_row = [&](int i) {
    const int row = jb.row0 + row_of(i), token = row / jb.g;
    return (int64_t)(jb.off + token) * p.Hq + hk * jb.g + (row - token * jb.g);
  };
#pragma unroll
  for (int i = 0; i < N; i++) {
    if (!live(i)) continue;
    const int orow = row_of(i);
    float mm = -INFINITY, ll = 0.f;
    f32x4 oo = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int x = 0; x < kF32Waves; x++) mm = fmaxf(mm, sh.ml[x][orow].x);
#pragma unroll
    for (int x = 0; x < kF32Waves; x++) {
      const float2 st = sh.ml[x][orow];
      const float wgt = state_weight(st.x, mm);
      ll += st.y * wgt;
      oo += *reinterpret_cast<const f32x4*>(&sh.o[x][orow * LS + c]) * wgt;
    }
    const int64_t grow = out_row(i);
    if (nsplit == 1) {
      *(CBL_GLOBAL f32x4*)((CBL_GLOBAL float*)p.out + grow * D + c) = oo / ll;
    } else {
      float* const pp = p.partial + (grow * p.nsplit + jb.split) * PS;
      put_pair(pp + c, oo[0], oo[1]);
      put_pair(pp + c + 2, oo[2], oo[3]);
      if (c == 0) put_pair(pp + D, mm, ll);
    }
  }
  if (nsplit == 1) return;
  // The stores are acknowledged before the ticket is drawn, so whoever completes the tile finds all of them in memory.
  asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
  __syncthreads();
  if (tid == 0) {
    CBL_GLOBAL uint32_t* const ticket = as_global(p.tickets) + ((int64_t)b * p.Hkv + hk) * jb.tiles + jb.rt;
    const uint32_t n = __hip_atomic_fetch_add(ticket, 1u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT) + 1;
    sh.last = n == (uint32_t)nsplit;
    if (n == (uint32_t)nsplit) __hip_atomic_store(ticket, 0u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);  // ready for the next launch
  }
  __syncthreads();
  if (!sh.last) return;
  auto merge = [&](auto batch) {   // (splits whose loads are in flight together)
    constexpr int BS = decltype(batch)::value;
#pragma unroll
    for (int i = 0; i < N; i++) {
      if (!live(i)) continue;
      const int64_t grow = out_row(i);
      const float* const part = p.partial + grow * p.nsplit * PS;
      float mm = -INFINITY, ll = 0.f;
      f32x4 oo = {0.f, 0.f, 0.f, 0.f};
      for (int t0 = 0; t0 < nsplit; t0 += BS) {
        float2 st[BS], x0[BS], x1[BS];
#pragma unroll
        for (int x = 0; x < BS; x++) {
          const float* const pp = part + (t0 + x < nsplit ? t0 + x : nsplit - 1) * PS;
          st[x] = get_pair(pp + D);
          x0[x] = get_pair(pp + c);
          x1[x] = get_pair(pp + c + 2);
        }
        float mn = mm;
#pragma unroll
        for (int x = 0; x < BS; x++) mn = fmaxf(mn, st[x].x);
        const float alpha = state_weight(mm, mn);
        oo *= alpha;
        ll *= alpha;
        mm = mn;
#pragma unroll
        for (int x = 0; x < BS; x++) {
          const bool more = t0 + x < nsplit;   // (not the last one once more)
          const float wgt = state_weight(st[x].x, mm);
          ll = more ? ll + st[x].y * wgt : ll;
          const f32x4 sum = oo + f32x4{x0[x].x, x0[x].y, x1[x].x, x1[x].y} * wgt;
#pragma unroll
          for (int e = 0; e < 4; e++) oo[e] = more ? sum[e] : oo[e];
        }
      }
      *(CBL_GLOBAL f32x4*)((CBL_GLOBAL float*)p.out + grow * D + c) = oo / ll;
    }
  };
  if (nsplit <= 8) merge(std::integral_constant<int, 8>{});
  else merge(std::integral_constant<int, 16>{});
}

hipError_t launch_attn_chunk_f32(hipStream_t st, const AttnParams& p, const SeqMeta& meta, const ChunkSplits& splits, int wgs) {
  const dim3 grid(wgs), block(64 * kF32Waves);
  if (p.D == 64 && p.tile_rows == 16) hipLaunchKernelGGL((k_chunk_f32<64, 1>), grid, block, 0, st, p, meta, splits);
  else if (p.D == 64) hipLaunchKernelGGL((k_chunk_f32<64, 2>), grid, block, 0, st, p, meta, splits);
  else if (p.tile_rows == 16) hipLaunchKernelGGL((k_chunk_f32<128, 1>), grid, block, 0, st, p, meta, splits);
  else hipLaunchKernelGGL((k_chunk_f32<128, 2>), grid, block, 0, st, p, meta, splits);
  return hipGetLastError();
}

}  // namespace cb
