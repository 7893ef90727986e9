// Attention of a chunk of new tokens over the cache (bf16, head_dim 64 or 128) on the matrix cores, gfx950 only.
//
// Token i of a sequence with S cached slots attends to slots 0 .. S + i: o = sum_j p_j v_j / sum_j p_j, p_j = exp(scale q.k_j - m).  The g query
// heads of a kv head share its K and V, so that a kv head's rows are g to a token, tokens one behind the other; tiles of up to 256
// rows are swept as the tree attention sweeps its own (cb_attn_wide.h), each up to its last token's slot.
//
// Probabilities are rounded to bf16, the matrix cores' type (half a step each, in the numerator and, the same, in the denominator); sums,
// statistics and partial states are in 32 bits.
#include "cb_attn_wide.h"
#include "cb_chunk.h"

namespace cb {

// Keys at or past `seen` (a query's own) or `kend` (the split's end) get -inf.
__device__ __forceinline__ void mask_chunk(floatx16& s, int key0, int seen, int kend, int h) {
  const int n = (seen < kend ? seen : kend) - key0 - 4 * h;
#pragma unroll
  for (int v = 0; v < 16; v++) s[v] = 8 * (v >> 2) + (v & 3) < n ? s[v] : -INFINITY;
}

// A value that a query must not see reaches its sum with weight 0, which hides it only if it is finite.  So units that some
// query of the tile does not see whole are added up with 0 in the place of infinities and NaN, and these, which hardly ever are there,
// separately to the queries that do see them.
__device__ __forceinline__ bf16x8 finite_only(bf16x8 a, bool& odd) {
  uintx4 x = __builtin_bit_cast(uintx4, a);
#pragma unroll
  for (int i = 0; i < 4; i++) {
    const bool lo = (x[i] & 0x7f80u) == 0x7f80u, hi = (x[i] & 0x7f800000u) == 0x7f800000u;
    odd |= lo || hi;
    x[i] = (lo ? 0u : x[i] & 0xffffu) | (hi ? 0u : x[i] & 0xffff0000u);
  }
  return __builtin_bit_cast(bf16x8, x);
}
template <int D>
__device__ __forceinline__ void add_odd_values(floatx16 (&o)[D / 32], const bf16x8& p0, const bf16x8& p1, uint32_t v_at, CB_LDS uint16_t* scratch, int l) {
  const int r = l & 31, h = l >> 5;
#pragma unroll
  for (int e = 0; e < 8; e++) {
    scratch[(8 * (e >> 2) + 4 * h + (e & 3)) * 32 + r] = __builtin_bit_cast(uint16_t, (__bf16)p0[e]);
    scratch[(16 + 8 * (e >> 2) + 4 * h + (e & 3)) * 32 + r] = __builtin_bit_cast(uint16_t, (__bf16)p1[e]);
  }
  asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
  for (int kk = 0; kk < kUnitKeys; kk++) {
    const float pk = __uint_as_float((uint32_t)scratch[kk * 32 + r] << 16);
#pragma unroll
    for (int dt = 0; dt < D / 32; dt++)
#pragma unroll
      for (int v = 0; v < 16; v++) {
        const int dim = 32 * dt + 8 * (v >> 2) + 4 * h + (v & 3);
        const uint32_t x = *(const CB_LDS uint16_t*)(v_at + kk * (2 * D) + (((dim >> 3) ^ swizzle_v<D, 32>(kk)) << 4) + (dim & 7) * 2);
        if ((x & 0x7f80u) == 0x7f80u && pk != 0.f) o[dt][v] += pk * __uint_as_float(x << 16);
      }
  }
}

// The sweep of one workgroup whose tile has RW row groups of R row tiles each, up to its output rows (a single split) or its
// partial state.
template <int D, bool PG, int R, int RW>
__device__ __forceinline__ void sweep_chunk(const AttnParams& p, const TileJob& jb, TileLds& sh, uint4* ring) {
  using Part = PartialLayout<D, 32, true>;
  using F = Feed<D, kWideWaves, 32>;
  constexpr int KW = kWideWaves / RW;    // key groups
  constexpr int NS = F::kSlots, PRO = F::kPrologue;
  constexpr int NPB = 2;                 // B operands of a unit's probabilities
  // (scores run one stage ahead of the softmax: two stages are resident while a third is requested)
  static_assert(3 * KW <= NS && KW <= PRO, "a stage is requested in full while the one before it is worked on");
  const int tid = threadIdx.x, w = __builtin_amdgcn_readfirstlane(tid >> 6), l = tid & 63;
  const int rw = w % RW, kw = w / RW;
  const int r = l & 31, h = l >> 5;
  const CB_GLOBAL uint16_t* gq = (const CB_GLOBAL uint16_t*)p.q;
  const int S = jb.S + jb.row0 / jb.g + 1;  // (every row sees the keys below)
  const int k0 = jb.k0, k1 = jb.k1;
  F ring_feed(p, jb, sh.bt, ring);
  WideFeed<D, PG> feed(ring_feed);
  // Everything the first stages need is requested up front, oldest first: the query rows (to registers), then K/V
  // units (to LDS).
  TileState<D> st[R];
  int seen[R];       // keys that the lane's queries see
  int64_t grow[R];   // their output rows (token * Hq + head), or -1 past the end
#pragma unroll
  for (int t = 0; t < R; t++) {
    int row = jb.row0 + (rw * R + t) * 32 + r;
    const bool valid = row < jb.M;
    row = valid ? row : jb.M - 1;
    const int token = row / jb.g;
    seen[t] = jb.S + token + 1;
    const int64_t gr = (int64_t)(jb.off + token) * p.Hq + jb.hk * jb.g + (row - token * jb.g);
    grow[t] = valid ? gr : -1;
    const CB_GLOBAL uintx4* qp = (const CB_GLOBAL uintx4*)(gq + gr * D);
#pragma unroll
    for (int ds = 0; ds < D / 16; ds++) st[t].q[ds] = __builtin_bit_cast(bf16x8, load_b128_untracked(qp + 2 * ds + h));
#pragma unroll
    for (int dt = 0; dt < D / 32; dt++)
#pragma unroll
      for (int v = 0; v < 16; v++) st[t].o[dt][v] = 0.f;
    st[t].lacc = floatx4{0.f, 0.f, 0.f, 0.f};
    st[t].mref = st[t].top = -INFINITY;
    st[t].nm = 0.f;
  }
  const bool has_rows = jb.row0 + rw * R * 32 < jb.M;
  const float c2 = p.scale * 1.4426950408889634f;  // softmax scale in the log2 domain

  const int nst = (k1 - k0 + kUnitKeys * KW - 1) / (kUnitKeys * KW);  // stages
  const int nu = nst * KW;                                            // units requested: whole stages
  feed.request_units(nu < PRO ? nu : PRO);
  ring_feed.wait_units(KW);
#pragma unroll
  for (int t = 0; t < R; t++)
#pragma unroll
    for (int ds = 0; ds < D / 16; ds++) {
      asm volatile("" : "+v"(st[t].q[ds]));  // (older than every unit)
#ifdef __HIP_DEVICE_COMPILE__
      if (R > 1) asm volatile("" : "+a"(st[t].q[ds]));  // (two tiles' queries live in accumulation registers)
#endif
    }

  // At the barrier in front of unit u NS - 2 units from u on have been requested.  It waits until those up to u + 3 have
  // landed; everybody is then done with those below u, whose places take the next requests.
  // (a split of fewer units waits for all of them at the first barrier)
  auto ready = [&] {
    wait_vmcnt<F::kReq * (NS - 6)>();
    bare_barrier();
  };
  auto first_ready = [&] {
    const int more = (nu < NS - 2 ? nu : NS - 2) - PRO;
    if (more > 0) feed.request_units(more);
    if (nu < NS - 2) wait_vmcnt<0>();
  };
  auto top = [&] {  // of a stage in the general loop, whose last reads may still be under way
    wait_vmcnt<F::kReq * (NS - 6)>();
    ring_barrier();
    feed.request_units(KW);
  };
  // this wave's stages whose units are all prefix and all inside the split (rounds down; may be negative: none)
  auto fast_stages = [&] {
    const int n = ((S < k1 ? S : k1) - k0 - kw * kUnitKeys) / (kUnitKeys * KW);
    return nst < n ? nst : n;
  };
  // Places in the ring, in bytes, of this wave's units of the current stage and the two behind it
  constexpr uint32_t kSlotBytes = F::kSlotBytes;
  auto next_place = [&](uint32_t x) { return x + KW * kSlotBytes >= NS * kSlotBytes ? x + KW * kSlotBytes - NS * kSlotBytes : x + KW * kSlotBytes; };
  uint32_t at = kw * kSlotBytes, at1 = next_place(at), at2 = next_place(at1);
  auto advance = [&] {
    at = at1;
    at1 = at2;
    at2 = next_place(at2);
  };
  const uint32_t lane_k = (uint32_t)(uintptr_t)(CB_LDS uint4*)ring + lane_k_byte<D>(l);
  const uint32_t lane_v = (uint32_t)(uintptr_t)(CB_LDS uint4*)ring + kSlotBytes / 2 + lane_v_byte<D>(l);
  const bf16x8 ones = half_ones(l);

  auto unit_scores = [&](int s, uint32_t place, floatx16 (&sc)[R]) {
    uint4 k[D / 16];
    read_k<D>(lane_k + place, k);
    scores<D, R>(k, st, sc);
    const int key0 = k0 + (s * KW + kw) * kUnitKeys;
    if (key0 + kUnitKeys > S || key0 + kUnitKeys > k1)
#pragma unroll
      for (int t = 0; t < R; t++) mask_chunk(sc[t], key0, seen[t], k1, h);
  };
  auto add_unit = [&](int s, const bf16x8 (&pb)[R][NPB], uint32_t place) {
    const uint32_t va = lane_v + place;
    const bool careful = k0 + (s * KW + kw) * kUnitKeys + kUnitKeys > S;  // (uniform)
    bool odd = false, odd_p = false;
    // (the denominator's MFMA has the probabilities of two queries in a column, one of them times 0)
#pragma unroll
    for (int t = 0; t < R; t++)
#pragma unroll
      for (int j = 0; j < NPB; j++)
        st[t].lacc = __builtin_amdgcn_mfma_f32_16x16x32_bf16(ones, careful ? finite_only(pb[t][j], odd_p) : pb[t][j], st[t].lacc, 0, 0, 0);
#pragma unroll
    for (int j = 0; j < 2; j++)
#pragma unroll
      for (int dt = 0; dt < D / 32; dt++) {
        bf16x8 a = read_v<D>(va, dt, j);
        if (careful) a = finite_only(a, odd);
#pragma unroll
        for (int t = 0; t < R; t++)
#pragma unroll
          for (int x = j; x < NPB; x += 2) st[t].o[dt] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(a, pb[t][x], st[t].o[dt], 0, 0, 0);
      }
    if (__builtin_expect(__builtin_amdgcn_ballot_w64(odd) != 0, 0)) {
      static_assert(sizeof(sh.anc) >= kWideWaves * kUnitKeys * 32 * 2, "");
#pragma unroll
      for (int t = 0; t < R; t++)
        add_odd_values<D>(st[t].o, pb[t][0], pb[t][1], (uint32_t)(uintptr_t)(CB_LDS uint4*)ring + place + kSlotBytes / 2, (CB_LDS uint16_t*)&sh.anc + w * (kUnitKeys * 32), l);
    }
  };
  auto sweep = [&] {
    floatx16 sc[R];
    bf16x8 pb[R][NPB];
    float mx[R];
    auto check = [&] {
      bool raise = mx[0] > st[0].top;  // (false for NaN)
      if (R > 1) raise |= mx[R - 1] > st[R - 1].top;
      if (__builtin_expect(__builtin_amdgcn_ballot_w64(raise) != 0, 0)) {
#pragma unroll
        for (int t = 0; t < R; t++) raise_reference<D>(st[t], mx[t], c2);
      }
    };
    auto maxima = [&](const floatx16 (&x)[R]) {
#pragma unroll
      for (int t = 0; t < R; t++) mx[t] = row_max(x[t]);
    };
    unit_scores(0, at, sc);
    maxima(sc);
    check();
    int s = 0;
    const int fast_end = fast_stages();
    floatx16 sd[R];
    uint4 k[D / 16];
    uintx4 pw[R][NPB];
    bf16x8 v[D / 32];
    // Stages whose units are all prefix, two at a time (the scores alternate between two sets of registers), the requests
    // spread over the steps (all at once they hold up the wave that makes them).  One barrier per two units.
    auto step = [&](const floatx16 (&from)[R], floatx16 (&to)[R], bool barrier) {  // stage s; from: its scores, to: those of stage s + 1
      if (barrier) ready();
      int64_t off[KW][F::kParts];
      uint32_t dst[KW];
#pragma unroll
      for (int x = 0; x < KW; x++) feed.next(off[x], dst[x]);
      if (KW > 1) read_k<D>(lane_k + at1, k);
      score_half<D, false, R, KW * F::kReq>(k, st, from, to, pw, lane_v + at, v, c2, [&](int i) {
        feed.request(i % F::kReq, off[i / F::kReq], dst[i / F::kReq]);
      });
      add_half<D, false, R, KW == 1>(k, lane_k + at2, lane_v + at, v, st, pw, to, mx, ones);
      check();
      advance();
      s++;
    };
    first_ready();
    if (s + 2 < fast_end) {
      if (KW == 1) {  // (K operands are a step ahead in registers)
        ready();
        read_k<D>(lane_k + at1, k);
      }
      do {
        step(sc, sd, true);
        step(sd, sc, KW > 1);
      } while (s + 2 < fast_end);
    }
    for (; s + 1 < nst; s++) {
      top();
      floatx16 sn[R];
      unit_scores(s + 1, at1, sn);
#pragma unroll
      for (int t = 0; t < R; t++) probs<D, false>(sc[t], st[t], c2, pb[t]);
      add_unit(s, pb, at);
      maxima(sn);
      check();
#pragma unroll
      for (int t = 0; t < R; t++) sc[t] = sn[t];
      advance();
    }
#pragma unroll
    for (int t = 0; t < R; t++) probs<D, false>(sc[t], st[t], c2, pb[t]);
    add_unit(s, pb, at);
  };
  if (has_rows) sweep();
  else {  // no rows of its own: it only brings its share, passing the same barriers
    int s = 0;
    first_ready();
    if constexpr (KW == 1) {
      const int fast_end = fast_stages();
      if (s + 2 < fast_end) ready();
      for (; s + 2 < fast_end; s += 2) {
        ready();
        feed.request_units(2);
      }
    }
    for (; s + 1 < nst; s++) top();
  }
  wait_vmcnt<0>();  // (the requests past the split's end, before the ring serves anything else)
  // With two key groups each finishes one half of the pieces: all park their accumulators and (mref, l) in the
  // ring, then each adds up the groups' for its own pieces.
  constexpr int P = Part::P, PP = P / KW;
  auto piece = [&](int t, int pc) {
    const floatx16& o = st[t].o[pc >> 2];
    return floatx4{o[4 * (pc & 3)], o[4 * (pc & 3) + 1], o[4 * (pc & 3) + 2], o[4 * (pc & 3) + 3]};
  };
  floatx4* const park = reinterpret_cast<floatx4*>(ring);
  float2* const park_ml = reinterpret_cast<float2*>(ring + kWideWaves * R * P * 64);
  if constexpr (KW > 1) {
    __syncthreads();  // every wave is done with the ring
    static_assert(kWideWaves * R * (P * 64 + 32) <= F::kRingVecs, "");
#pragma unroll
    for (int t = 0; t < R; t++) {
#pragma unroll
      for (int pc = 0; pc < P; pc++) park[((w * R + t) * P + pc) * 64 + l] = piece(t, pc);  // (w = kw * RW + rw)
      park_ml[(w * R + t) * 64 + l] = float2{st[t].mref, st[t].lacc[0]};
    }
    __syncthreads();
  }
#pragma unroll
  for (int t = 0; t < R; t++) {
    floatx4 f[PP];
    float lsum, mfin;
    if constexpr (KW > 1) {
      float2 ml[KW];
      mfin = -INFINITY;
#pragma unroll
      for (int k = 0; k < KW; k++) {
        ml[k] = park_ml[((k * RW + rw) * R + t) * 64 + l];
        mfin = fmaxf(mfin, ml[k].x);
      }
      const float mu = (mfin == -INFINITY) ? 0.f : mfin;
      lsum = 0.f;
#pragma unroll
      for (int i = 0; i < PP; i++) f[i] = floatx4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int k = 0; k < KW; k++) {
        const float wt = __builtin_amdgcn_exp2f((ml[k].x - mu) * c2);
        lsum += ml[k].y * wt;
#pragma unroll
        for (int i = 0; i < PP; i++) f[i] += park[(((k * RW + rw) * R + t) * P + kw * PP + i) * 64 + l] * wt;
      }
    } else {
      lsum = st[t].lacc[0];
      mfin = st[t].mref;
#pragma unroll
      for (int i = 0; i < PP; i++) f[i] = piece(t, i);
    }
    write_rows<D, 32, true, PP>(p, jb, rw * R + t, grow[t], f, kw * PP, mfin, lsum, c2, kw == 0, l);
  }
}

template <int D, bool PG>
__global__ __launch_bounds__(64 * kWideWaves, 1) void k_chunk(AttnParams p_arg, SeqMeta meta) {
  const SeqMetaLanes ml = seq_meta_prefetch(meta);
  __shared__ __align__(1024) uint4 ring[Feed<D, kWideWaves, 32>::kRingVecs];
  __shared__ TileLds sh;
  AttnParams p = p_arg;
  pin_args(p);
  TileJob jb;
  if (!chunk_job(p, ml, blockIdx.x, jb)) return;
  const int rows = jb.M - jb.row0 < p.tile_rows ? jb.M - jb.row0 : p.tile_rows;
  if (rows <= 64) sweep_chunk<D, PG, 1, 2>(p, jb, sh, ring);
  else if (rows <= 128) sweep_chunk<D, PG, 1, 4>(p, jb, sh, ring);
  else sweep_chunk<D, PG, 2, 4>(p, jb, sh, ring);
  if (jb.nsplit > 1) split_merge<D, 32, true, kWideWaves, 256, false>(p, jb, p.tile_rows, sh, nullptr, [] {});
}

int64_t chunk_partial_bytes(int D, int64_t total, int Hq, int Hkv, int batch) {
  const int64_t tiles = total * Hq / 32 + (int64_t)(Hkv + 1) * batch + 1;  // (block_tile0)
  return tiles * (D == 64 ? PartialLayout<64, 32, true>::kBytes : PartialLayout<128, 32, true>::kBytes);
}

hipError_t launch_attn_chunk(hipStream_t st, const AttnParams& p, const SeqMeta& meta, int wgs) {
  const dim3 grid(wgs), block(64 * kWideWaves);
  const bool paged = p.kv.block_size > 0;
  if (p.D == 64 && paged) hipLaunchKernelGGL((k_chunk<64, true>), grid, block, 0, st, p, meta);
  else if (p.D == 64) hipLaunchKernelGGL((k_chunk<64, false>), grid, block, 0, st, p, meta);
  else if (paged) hipLaunchKernelGGL((k_chunk<128, true>), grid, block, 0, st, p, meta);
  else hipLaunchKernelGGL((k_chunk<128, false>), grid, block, 0, st, p, meta);
  return hipGetLastError();
}

}  // namespace cb
