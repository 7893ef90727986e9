// Attention of a chunk of new tokens over the cache (bf16, head_dim 64 or 128) on the matrix cores, gfx950 only.
//
// Token i of a sequence with S cached slots attends to slots 0 .. S + i: o = sum_j p_j v_j / sum_j p_j, p_j = exp(scale q.k_j - m).  The g query
// heads of a kv head share its K and V, so that a kv head's rows are g to a token, tokens one behind the other; tiles of up to 256
// rows are swept as the tree attention sweeps its own (cb_attn_wide.h), each up to its last token's slot.
//
// Probabilities are rounded to bf16, the matrix cores' type (half a step each, in the numerator and, the same, in the denominator); sums,
// statistics and partial states are in 32 bits.
//
// What bounds it, at 32/8 heads of 128: long sweeps the matrix cores beside the vector units, at the 1.9 to 2.1 GHz that this power allows (4096 tokens
// behind 28672 1.82 ms, 1130 TFLOP/s; a library product's rate is 1250; a compute unit's matrix cores are busy 56% of its time, its vector units 47%, both
// 24%); single tokens reading the cache (16 sequences of up to 16384 105 us, 5.0 TB/s); short chunks a launch, a workgroup's start and the way of a split's state through memory (1024 tokens from
// the first 24 us).  Hence three tiles, for a rule by the host: of 64 rows, whose workgroup has the whole ring of LDS for keys on their way, of
// 128, two to a compute unit, and of 256, which read an operand from LDS for 64 rows.
#include "cb_attn_wide.h"
#include "cb_chunk.h"

namespace cb {

// Keys at or past `seen` (a query's own) or `kend` (the split's end) get -inf.
__device__ __forceinline__ void mask_chunk(floatx16& s, int key0, int seen, int kend, int h) {
  const int n = (seen < kend ? seen : kend) - key0 - 4 * h;
#pragma unroll
  for (int v = 0; v < 16; v++) s[v] = 8 * (v >> 2) + (v & 3) < n ? s[v] : -INFINITY;
}

// A value that a query must not see, or a split's last one in the places behind it, reaches a sum with weight 0, which hides it only if it is finite;
// and the denominator's MFMA has the probabilities of two queries in a column, one of them times 0, so that a query whose scores are not finite
// reaches another one's sum.  What is no number stays none in a sum, so every tile looks at its sums when its sweep is through, and one that has
// infinities or NaN is swept again with care: with 0 in the place of those, and values of these added up separately for the queries that do see them.
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
// p0, p1: the lane's probabilities (B operands); v_at: the unit's values in LDS; sees: how many of its keys the lane's query sees.  One whose probability is
// 0 in 32 bits has a positive weight all the same, and an infinity or NaN times that is what it is.
template <int D>
__device__ __forceinline__ void add_odd_values(floatx16 (&o)[D / 32], const bf16x8& p0, const bf16x8& p1, uint32_t v_at, int sees, int l) {
  const int r = l & 31, h = l >> 5;
  const uintx4 x0 = __builtin_bit_cast(uintx4, p0), x1 = __builtin_bit_cast(uintx4, p1);
  for (int kk = 0; kk < kUnitKeys; kk++) {
    // key 16 j + 8 (e / 4) + 4 h + e % 4 is element e of operand j of the lane in half h
    const int at = (kk >> 4) * 4 + (kk >> 3 & 1) * 2 + (kk >> 1 & 1);
    uint32_t pair = x0[0];
#pragma unroll
    for (int i = 1; i < 8; i++) pair = at == i ? (i < 4 ? x0[i & 3] : x1[i & 3]) : pair;
    pair = (uint32_t)__shfl((int)pair, (kk >> 2 & 1) * 32 + r, 64);
    const float pk = __uint_as_float(kk & 1 ? pair & 0xffff0000u : pair << 16);
#pragma unroll
    for (int dt = 0; dt < D / 32; dt++)
#pragma unroll
      for (int v = 0; v < 16; v++) {
        const int dim = 32 * dt + 8 * (v >> 2) + 4 * h + (v & 3);
        const uint32_t x = *(const CB_LDS uint16_t*)(v_at + kk * (2 * D) + (((dim >> 3) ^ swizzle_v<D, 32>(kk)) << 4) + (dim & 7) * 2);
        if ((x & 0x7f80u) == 0x7f80u && kk < sees) o[dt][v] += (pk == 0.f ? 1.f : pk) * __uint_as_float(x << 16);
      }
  }
}

// Whether some wavefront's sums have infinities or NaN.  A barrier.
template <int D, int R>
__device__ __forceinline__ bool any_odd(const TileState<D> (&st)[R], int (&odd)[kWideWaves], int w, int l) {
  float x[4] = {};  // (times 0 and added up: 0 or NaN; four chains)
#pragma unroll
  for (int t = 0; t < R; t++) {
    x[t] = fmaf(st[t].lacc[0], 0.f, x[t]);
#pragma unroll
    for (int dt = 0; dt < D / 32; dt++)
#pragma unroll
      for (int v = 0; v < 16; v++) x[v & 3] = fmaf(st[t].o[dt][v], 0.f, x[v & 3]);
  }
  const bool mine = __builtin_amdgcn_ballot_w64((x[0] + x[1]) + (x[2] + x[3]) != 0.f) != 0;
  if (l == 0) odd[w] = mine;
  __syncthreads();
  int any = 0;
#pragma unroll
  for (int i = 0; i < kWideWaves; i++) any |= odd[i];
  return any != 0;
}

// Tiles of up to 64 rows, two row groups of a row tile each and two wavefronts to a group, which take the units in turn: the sweep of one workgroup
// up to its output rows (a single split) or its partial state.  Without CARE it returns true where the tile has to be swept with.
template <int D, bool PG, bool CARE>
__device__ __forceinline__ bool sweep_few(const AttnParams& p, const TileJob& jb, TileLds& sh, int (&odd)[kWideWaves], uint4* ring) {
  using Part = PartialLayout<D, 32, true>;
  using F = Feed<D, kWideWaves, 32>;
  constexpr int R = 1, RW = 2, KW = kWideWaves / RW;   // row tiles of a row group, row groups, key groups
  constexpr int NS = F::kSlots, PRO = F::kPrologue;
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
    for (int ds = 0; ds < D / 16; ds++) asm volatile("" : "+v"(st[t].q[ds]));  // (older than every unit)

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
  // whether some query may not see some key of the stage, or the split ends in it (uniform in the workgroup)
  const int whole_end = S < k1 ? S : k1;
  auto masked = [&](int s) { return k0 + (s + 1) * KW * kUnitKeys > whole_end; };
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

  auto mask = [&](int s, floatx16 (&sc)[R]) {
    if (!masked(s)) return;
#pragma unroll
    for (int t = 0; t < R; t++) mask_chunk(sc[t], k0 + (s * KW + kw) * kUnitKeys, seen[t], k1, h);
  };
  auto sweep = [&] {
    floatx16 sc[R];
    float mx[R];
    auto check = [&] {
      const bool raise = mx[0] > st[0].top;  // (false for NaN)
      if (__builtin_expect(__builtin_amdgcn_ballot_w64(raise) != 0, 0)) {
#pragma unroll
        for (int t = 0; t < R; t++) raise_reference<D>(st[t], mx[t], c2);
      }
    };
    floatx16 sd[R];
    uint4 k[D / 16];
    uintx4 pw[R][2];
    bf16x8 v[D / 32];
    read_k<D>(lane_k + at, k);
    scores<D, R>(k, st, sc);
    mask(0, sc);
#pragma unroll
    for (int t = 0; t < R; t++) mx[t] = row_max(sc[t]);
    check();
    int s = 0;
    // A step: the scores of stage s + 1 beside the exponentials of stage s, then its values; two at a time (the scores alternate between two
    // sets of registers), the requests spread over the steps (all at once they hold up the wave that makes them).
    auto step = [&](const floatx16 (&from)[R], floatx16 (&to)[R], bool masks) {  // from: the scores of stage s, to: those of stage s + 1
      ready();
      int64_t off[KW][F::kParts];
      uint32_t dst[KW];
#pragma unroll
      for (int x = 0; x < KW; x++) feed.next(off[x], dst[x]);
      read_k<D>(lane_k + at1, k);
      score_half<D, false, R, KW * F::kReq>(k, st, from, to, pw, lane_v + at, v, c2, [&](int i) {
        feed.request(i % F::kReq, off[i / F::kReq], dst[i / F::kReq]);
      });
      if (masks) mask(s + 1, to);
      add_half<D, false, R, false>(k, lane_k + at2, lane_v + at, v, st, pw, to, mx, ones);
      check();
      advance();
      s++;
    };
    first_ready();
    while (s + 2 < nst && !masked(s + 2)) {
      step(sc, sd, false);
      step(sd, sc, false);
    }
    bf16x8 pb[R][2];
    auto add_unit = [&] {
      const uint32_t va = lane_v + at;
#pragma unroll
      for (int t = 0; t < R; t++)
#pragma unroll
        for (int j = 0; j < 2; j++) st[t].lacc = __builtin_amdgcn_mfma_f32_16x16x32_bf16(ones, pb[t][j], st[t].lacc, 0, 0, 0);
#pragma unroll
      for (int j = 0; j < 2; j++)
#pragma unroll
        for (int dt = 0; dt < D / 32; dt++) {
          const bf16x8 a = read_v<D>(va, dt, j);
#pragma unroll
          for (int t = 0; t < R; t++) st[t].o[dt] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(a, pb[t][j], st[t].o[dt], 0, 0, 0);
        }
    };
    // Stages with masks, one at a time.
    while (s + 1 < nst) {
      step(sc, sd, true);
#pragma unroll
      for (int t = 0; t < R; t++) sc[t] = sd[t];
    }
#pragma unroll
    for (int t = 0; t < R; t++) probs<D, false>(sc[t], st[t], c2, pb[t]);
    add_unit();
  };
  // The same with care, a stage at a time.
  auto careful_sweep = [&] {
    auto top = [&] {  // (the stage's last reads may still be under way)
      wait_vmcnt<F::kReq * (NS - 6)>();
      ring_barrier();
      feed.request_units(KW);
    };
    first_ready();
    if (!has_rows) {
      for (int s = 0; s + 1 < nst; s++) top();
      return;
    }
    floatx16 sc[R];
    bf16x8 pb[R][2];
    for (int s = 0; s < nst; s++) {
      if (s > 0) {
        advance();
        top();
      }
      uint4 k[D / 16];
      read_k<D>(lane_k + at, k);
      scores<D, R>(k, st, sc);
      mask(s, sc);
      bool raise = false, odd_v = false, odd_p = false;
      float mx[R];
#pragma unroll
      for (int t = 0; t < R; t++) {
        mx[t] = row_max(sc[t]);
        raise |= mx[t] > st[t].top;
      }
      if (__builtin_amdgcn_ballot_w64(raise) != 0) {
#pragma unroll
        for (int t = 0; t < R; t++) raise_reference<D>(st[t], mx[t], c2);
      }
#pragma unroll
      for (int t = 0; t < R; t++) {
        probs<D, false>(sc[t], st[t], c2, pb[t]);
#pragma unroll
        for (int j = 0; j < 2; j++) st[t].lacc = __builtin_amdgcn_mfma_f32_16x16x32_bf16(ones, finite_only(pb[t][j], odd_p), st[t].lacc, 0, 0, 0);
      }
#pragma unroll
      for (int j = 0; j < 2; j++)
#pragma unroll
        for (int dt = 0; dt < D / 32; dt++) {
          const bf16x8 a = finite_only(read_v<D>(lane_v + at, dt, j), odd_v);
#pragma unroll
          for (int t = 0; t < R; t++) st[t].o[dt] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(a, pb[t][j], st[t].o[dt], 0, 0, 0);
        }
      if (__builtin_amdgcn_ballot_w64(odd_v) != 0) {
#pragma unroll
        for (int t = 0; t < R; t++) add_odd_values<D>(st[t].o, pb[t][0], pb[t][1], (uint32_t)(uintptr_t)(CB_LDS uint4*)ring + at + kSlotBytes / 2, (seen[t] < k1 ? seen[t] : k1) - k0 - (s * KW + kw) * kUnitKeys, l);
      }
    }
  };
  if constexpr (CARE) careful_sweep();
  else if (has_rows) sweep();
  else {  // no rows of its own: it only brings its share, passing the same barriers
    first_ready();
    int s = 0;
    for (; s + 1 < nst; s++) {
      ready();
      feed.request_units(KW);
      advance();
    }
  }
  wait_vmcnt<0>();  // (the requests past the split's end, before the ring serves anything else)
  if (CARE) __syncthreads();  // every wave is done with the ring
  else if (any_odd<D>(st, odd, w, l)) return true;
  // With two key groups each finishes one half of the pieces: all park their accumulators and (mref, l) in the
  // ring, then each adds up the groups' for its own pieces.
  constexpr int P = Part::P, PP = P / KW;
  auto piece = [&](int t, int pc) {
    const floatx16& o = st[t].o[pc >> 2];
    return floatx4{o[4 * (pc & 3)], o[4 * (pc & 3) + 1], o[4 * (pc & 3) + 2], o[4 * (pc & 3) + 3]};
  };
  floatx4* const park = reinterpret_cast<floatx4*>(ring);
  float2* const park_ml = reinterpret_cast<float2*>(ring + kWideWaves * R * P * 64);
  static_assert(kWideWaves * R * (P * 64 + 32) <= F::kRingVecs, "");
#pragma unroll
  for (int t = 0; t < R; t++) {
#pragma unroll
    for (int pc = 0; pc < P; pc++) park[((w * R + t) * P + pc) * 64 + l] = piece(t, pc);  // (w = kw * RW + rw)
    park_ml[(w * R + t) * 64 + l] = float2{st[t].mref, st[t].lacc[0]};
  }
  __syncthreads();
#pragma unroll
  for (int t = 0; t < R; t++) {
    floatx4 f[PP];
    float2 ml[KW];
    float lsum = 0.f, mfin = -INFINITY;
#pragma unroll
    for (int k = 0; k < KW; k++) {
      ml[k] = park_ml[((k * RW + rw) * R + t) * 64 + l];
      mfin = fmaxf(mfin, ml[k].x);
    }
    const float mu = (mfin == -INFINITY) ? 0.f : mfin;
#pragma unroll
    for (int i = 0; i < PP; i++) f[i] = floatx4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int k = 0; k < KW; k++) {
      const float wt = __builtin_amdgcn_exp2f((ml[k].x - mu) * c2);
      lsum += ml[k].y * wt;
#pragma unroll
      for (int i = 0; i < PP; i++) f[i] += park[(((k * RW + rw) * R + t) * P + kw * PP + i) * 64 + l] * wt;
    }
    write_rows<D, 32, true, PP>(p, jb, rw * R + t, grow[t], f, kw * PP, mfin, lsum, c2, kw == 0, l);
  }
  return false;
}

// Tiles of up to 256 rows in long sweeps, four wavefronts of two row tiles, one workgroup to a compute unit: an operand read from LDS serves 64
// rows.  Units that some query does not see whole, few there, are taken one at a time and with care in any case (without, the compiler moves the sums
// between register files in the other units' loop: 4096 tokens behind 28672 2170 us, and 1820).  Without CARE it returns true where all units have to be.
template <int D, bool PG, bool CARE>
__device__ __forceinline__ bool sweep_tall(const AttnParams& p, const TileJob& jb, TileLds& sh, int (&odd)[kWideWaves], uint4* ring) {
  constexpr int R = 2;
  using Part = PartialLayout<D, 32, true>;
  using F = Feed<D, kWideWaves, 32>;
  constexpr int NS = F::kSlots, PRO = F::kPrologue;
  const int tid = threadIdx.x, w = __builtin_amdgcn_readfirstlane(tid >> 6), l = tid & 63;
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
    int row = jb.row0 + (w * R + t) * 32 + r;
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
  const bool has_rows = jb.row0 + w * R * 32 < jb.M;
  const float c2 = p.scale * 1.4426950408889634f;  // softmax scale in the log2 domain

  const int nst = (k1 - k0 + kUnitKeys - 1) / kUnitKeys;  // stages
  feed.request_units(nst < PRO ? nst : PRO);
  ring_feed.wait_units(1);
#pragma unroll
  for (int t = 0; t < R; t++)
#pragma unroll
    for (int ds = 0; ds < D / 16; ds++) {
      asm volatile("" : "+v"(st[t].q[ds]));  // (older than every unit)
#ifdef __HIP_DEVICE_COMPILE__
      asm volatile("" : "+a"(st[t].q[ds]));  // (two tiles' queries live in accumulation registers)
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
    const int more = (nst < NS - 2 ? nst : NS - 2) - PRO;
    if (more > 0) feed.request_units(more);
    if (nst < NS - 2) wait_vmcnt<0>();
  };
  auto top = [&] {  // of a stage in the general loop, whose last reads may still be under way
    wait_vmcnt<F::kReq * (NS - 6)>();
    ring_barrier();
    feed.request_units(1);
  };
  // this wave's stages whose units are all prefix and all inside the split (rounds down; may be negative: none)
  auto fast_stages = [&] {
    if (CARE) return 0;
    const int n = ((S < k1 ? S : k1) - k0) / kUnitKeys;
    return nst < n ? nst : n;
  };
  // Places in the ring, in bytes, of this wave's units of the current stage and the two behind it
  constexpr uint32_t kSlotBytes = F::kSlotBytes;
  auto next_place = [&](uint32_t x) { return x + kSlotBytes == NS * kSlotBytes ? 0 : x + kSlotBytes; };
  uint32_t at = 0, at1 = next_place(at), at2 = next_place(at1);
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
    const int key0 = k0 + s * kUnitKeys;
    if (key0 + kUnitKeys > S || key0 + kUnitKeys > k1)
#pragma unroll
      for (int t = 0; t < R; t++) mask_chunk(sc[t], key0, seen[t], k1, h);
  };
  auto add_unit = [&](int s, const bf16x8 (&pb)[R][2], uint32_t place) {
    const uint32_t va = lane_v + place;
    const bool careful = CARE || k0 + s * kUnitKeys + kUnitKeys > S;  // (uniform)
    bool odd_v = false, odd_p = false;
#pragma unroll
    for (int t = 0; t < R; t++)
#pragma unroll
      for (int j = 0; j < 2; j++)
        st[t].lacc = __builtin_amdgcn_mfma_f32_16x16x32_bf16(ones, careful ? finite_only(pb[t][j], odd_p) : pb[t][j], st[t].lacc, 0, 0, 0);
#pragma unroll
    for (int j = 0; j < 2; j++)
#pragma unroll
      for (int dt = 0; dt < D / 32; dt++) {
        bf16x8 a = read_v<D>(va, dt, j);
        if (careful) a = finite_only(a, odd_v);
#pragma unroll
        for (int t = 0; t < R; t++) st[t].o[dt] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(a, pb[t][j], st[t].o[dt], 0, 0, 0);
      }
    if (__builtin_expect(__builtin_amdgcn_ballot_w64(odd_v) != 0, 0)) {
#pragma unroll
      for (int t = 0; t < R; t++) add_odd_values<D>(st[t].o, pb[t][0], pb[t][1], (uint32_t)(uintptr_t)(CB_LDS uint4*)ring + place + kSlotBytes / 2, (seen[t] < k1 ? seen[t] : k1) - k0 - s * kUnitKeys, l);
    }
  };
  auto sweep = [&] {
    floatx16 sc[R];
    bf16x8 pb[R][2];
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
    uintx4 pw[R][2];
    bf16x8 v[D / 32];
    // Stages whose units are all prefix, two at a time (the scores alternate between two sets of registers), the requests
    // spread over the steps (all at once they hold up the wave that makes them).  One barrier per two units.
    auto step = [&](const floatx16 (&from)[R], floatx16 (&to)[R], bool barrier) {  // stage s; from: its scores, to: those of stage s + 1
      if (barrier) ready();
      int64_t off[F::kParts];
      uint32_t dst;
      feed.next(off, dst);
      score_half<D, false, R, F::kReq>(k, st, from, to, pw, lane_v + at, v, c2, [&](int i) {
        feed.request(i, off, dst);
      });
      add_half<D, false, R, true>(k, lane_k + at2, lane_v + at, v, st, pw, to, mx, ones);
      check();
      advance();
      s++;
    };
    first_ready();
    if (s + 2 < fast_end) {
      ready();  // (K operands are a step ahead in registers)
      read_k<D>(lane_k + at1, k);
      do {
        step(sc, sd, true);
        step(sd, sc, false);
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
    const int fast_end = fast_stages();
    if (s + 2 < fast_end) ready();
    for (; s + 2 < fast_end; s += 2) {
      ready();
      feed.request_units(2);
    }
    for (; s + 1 < nst; s++) top();
  }
  wait_vmcnt<0>();  // (the requests past the split's end, before the ring serves anything else)
  if (!CARE && any_odd<D>(st, odd, w, l)) return true;
#pragma unroll
  for (int t = 0; t < R; t++) {
    floatx4 f[Part::P];
#pragma unroll
    for (int pc = 0; pc < Part::P; pc++) {
      const floatx16& o = st[t].o[pc >> 2];
      f[pc] = floatx4{o[4 * (pc & 3)], o[4 * (pc & 3) + 1], o[4 * (pc & 3) + 2], o[4 * (pc & 3) + 3]};
    }
    write_rows<D, 32, true, Part::P>(p, jb, w * R + t, grow[t], f, 0, st[t].mref, st[t].lacc[0], c2, true, l);
  }
  return false;
}

// Tiles of up to 128 rows, four wavefronts of 32 rows, two workgroups to a compute unit: the one's start, tail and barriers are behind
// the other's sweep.  K and V have rings of their own, a unit's K being read a step before its V, so that 72 KiB hold what is worked on
// and two units that are under way.
template <int D>
struct ManyLds {
  static constexpr int kK = 5, kV = 4;                          // units
  static constexpr int kBytes = kUnitKeys * D * 2;              // of a unit's K, or V
  uint4 ring[(kK + kV) * kBytes / 16];
  int bt[kBtLds];
  int flag;
  int odd[kWideWaves];
};

// The memory side: K of a unit is requested two steps before its V, whose addresses wait in registers until then.
template <int D, bool PG>
struct ManyFeed {
  using F = Feed<D, kWideWaves, 32>;
  using L = ManyLds<D>;
  static constexpr int P = F::kParts, RPR = F::RPR;
  static_assert(F::kReq == 2 * P, "a group is a request for K and one for V");
  F& f;
  int key[P];                            // the lane's row in the next unit's groups, at most the split's last key
  const int last;
  const CB_GLOBAL char *kb[P], *vb[P];   // what the row's offset is added to
  uint32_t k_place = 0, v_place = 0;     // of the next unit in the rings, bytes
  int blk[P];                            // paged: the rows' entries of the block table
  int64_t off[P], later[2][P];           // offsets of the unit whose K is next, and of the two whose V are
  __device__ __forceinline__ explicit ManyFeed(F& feed) : f(feed), last(feed.jb.k1 - 1) {
    const AttnParams& p = f.p;
    const int lr = f.l / F::VPR, lc = f.l % F::VPR;
    const int64_t head = ((PG ? 0 : (int64_t)f.jb.b * p.kv.seq_stride) + (int64_t)f.jb.hk * p.kv.head_stride) * 2;
#pragma unroll
    for (int i = 0; i < P; i++) {
      const int rr = f.part_row(i) + lr;
      key[i] = f.jb.k0 + rr;
      key[i] = key[i] < last ? key[i] : last;
      kb[i] = f.kbase + head + (lc ^ swizzle_k<D>(rr)) * 16;
      vb[i] = f.vbase + head + (lc ^ swizzle_v<D, 32>(rr)) * 16;
      blk[i] = 0;
      later[0][i] = later[1][i] = 0;
    }
    if (PG) look_up();
  }
  __device__ __forceinline__ void look_up() {
#pragma unroll
    for (int i = 0; i < P; i++) blk[i] = f.bt[((key[i] >> f.ka.bs_shift) - f.ka.bt_first) & (kBtLds - 1)];
  }
  // The next unit's offsets, and on to the one behind it (whose table entries are asked for here and looked at a step later).
  __device__ __forceinline__ void next() {
    const KvAddr& a = f.p.kv;
    if (PG) {
      if (f.long_slice) f.bt_ahead(f.requested);
#pragma unroll
      for (int i = 0; i < P; i++) {
        int b = blk[i];
        b = b < 0 ? 0 : (b >= (int)a.num_blocks ? (int)a.num_blocks - 1 : b);
        off[i] = (int64_t)(uint64_t)(uint32_t)b * (a.seq_stride * 2) + (int64_t)((uint64_t)(uint32_t)(key[i] & (a.block_size - 1)) * (uint32_t)f.ts2);
      }
    } else {
#pragma unroll
      for (int i = 0; i < P; i++) off[i] = (int64_t)((uint64_t)(uint32_t)key[i] * (uint32_t)f.ts2);
    }
#pragma unroll
    for (int i = 0; i < P; i++) {
      key[i] += kUnitKeys;
      key[i] = key[i] < last ? key[i] : last;
    }
    if (PG) look_up();
    f.requested++;
  }
  __device__ __forceinline__ uint32_t lds_at() const { return f.part_row(0) * (2 * D) + __builtin_amdgcn_readfirstlane((uint32_t)(uintptr_t)(CB_LDS uint4*)f.ring); }
  // request i of a step's 2 P (a constant): K's groups, then those of the V that is due
  __device__ __forceinline__ void request(int i) const {
    if (i < P) lds_dma_b128_at(kb[i] + off[i], lds_at() + k_place + i * (RPR * 2 * D));
    else lds_dma_b128_at(vb[i - P] + later[0][i - P], lds_at() + v_place + L::kK * L::kBytes + (i - P) * (RPR * 2 * D));
  }
  __device__ __forceinline__ void requested(bool k, bool v) {  // which of the two a step has made
    if (k) k_place = k_place + L::kBytes == L::kK * L::kBytes ? 0 : k_place + L::kBytes;
    if (v) v_place = v_place + L::kBytes == L::kV * L::kBytes ? 0 : v_place + L::kBytes;
#pragma unroll
    for (int i = 0; i < P; i++) {
      later[0][i] = later[1][i];
      later[1][i] = off[i];
    }
  }
  __device__ __forceinline__ void request_step(bool v = true) {
    next();
#pragma unroll
    for (int i = 0; i < 2 * P; i++)
      if (v || i < P) request(i);
    requested(true, v);
  }
};

// Up to the tile's output rows or its partial state.  Without CARE it returns true where the tile has to be swept with.
template <int D, bool PG, bool CARE>
__device__ __forceinline__ bool sweep_many(const AttnParams& p, const TileJob& jb, ManyLds<D>& sh) {
  using Part = PartialLayout<D, 32, true>;
  using F = Feed<D, kWideWaves, 32>;
  using L = ManyLds<D>;
  constexpr int R = 1;  // row tiles of a wavefront
  const int tid = threadIdx.x, w = __builtin_amdgcn_readfirstlane(tid >> 6), l = tid & 63, r = l & 31, h = l >> 5;
  const CB_GLOBAL uint16_t* gq = (const CB_GLOBAL uint16_t*)p.q;
  const int S = jb.S + jb.row0 / jb.g + 1;  // (every row sees the keys below)
  const int k0 = jb.k0, k1 = jb.k1;
  F ring_feed(p, jb, sh.bt, sh.ring);
  ManyFeed<D, PG> feed(ring_feed);
  TileState<D> st[R];
  int seen[R];       // keys that the lane's queries see
  int64_t grow[R];   // their output rows (token * Hq + head), or -1 past the end
#pragma unroll
  for (int t = 0; t < R; t++) {
    int row = jb.row0 + (w * R + t) * 32 + r;
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
  const bool has_rows = jb.row0 + w * R * 32 < jb.M;
  const float c2 = p.scale * 1.4426950408889634f;  // softmax scale in the log2 domain
  const int nst = (k1 - k0 + kUnitKeys - 1) / kUnitKeys;
  // K of five units and V of three (past the split's end: its last key); the first two units' K have landed at the first barrier
  feed.request_step(false);
  feed.request_step(false);
  for (int u = 0; u < 3; u++) feed.request_step();
  wait_vmcnt<3 * F::kReq>();
  ring_barrier();
#pragma unroll
  for (int t = 0; t < R; t++)
#pragma unroll
    for (int ds = 0; ds < D / 16; ds++) asm volatile("" : "+v"(st[t].q[ds]));  // (older than every unit)
  // At the barrier of step s K up to unit s + 4 and V up to s + 2 have been requested, and K up to s + 2 and V up to s have landed; everybody is
  // done with K(s) and V(s - 1) (reads of K(s + 1) may be under way), whose places take K(s + 5) and V(s + 3).
  auto ready = [&] {
    wait_vmcnt<2 * F::kReq>();
    bare_barrier();
  };
  const int whole_end = S < k1 ? S : k1;
  auto masked = [&](int s) { return k0 + (s + 1) * kUnitKeys > whole_end; };
  const uint32_t ring = (uint32_t)(uintptr_t)(CB_LDS uint4*)sh.ring, vring = ring + L::kK * L::kBytes;
  const uint32_t lane_k = ring + lane_k_byte<D>(l), lane_v = vring + lane_v_byte<D>(l);
  const bf16x8 ones = half_ones(l);
  uint32_t k_at = 0, v_at = 0;  // places of the K that is read next and of V(s)
  auto advance_k = [&] { k_at = k_at + L::kBytes == L::kK * L::kBytes ? 0 : k_at + L::kBytes; };
  auto advance_v = [&] { v_at = v_at + L::kBytes == L::kV * L::kBytes ? 0 : v_at + L::kBytes; };
  auto mask = [&](int s, floatx16 (&sc)[R]) {
    if (!masked(s)) return;
#pragma unroll
    for (int t = 0; t < R; t++) mask_chunk(sc[t], k0 + s * kUnitKeys, seen[t], k1, h);
  };
  auto check = [&](const float (&mx)[R]) {
    bool raise = mx[0] > st[0].top;  // (false for NaN)
    if (R > 1) raise |= mx[R - 1] > st[R - 1].top;
    if (__builtin_expect(__builtin_amdgcn_ballot_w64(raise) != 0, 0)) {
#pragma unroll
      for (int t = 0; t < R; t++) raise_reference<D>(st[t], mx[t], c2);
    }
  };
  auto sweep = [&] {
    floatx16 sc[R], sd[R];
    float mx[R];
    uint4 k[D / 16];
    uintx4 pw[R][2];
    bf16x8 v[D / 32];
    read_k<D>(lane_k, k);
    scores<D, R>(k, st, sc);
    mask(0, sc);
#pragma unroll
    for (int t = 0; t < R; t++) mx[t] = row_max(sc[t]);
    check(mx);
    advance_k();
    read_k<D>(lane_k + k_at, k);
    advance_k();
    // A step: the scores of unit s + 1 beside the exponentials of unit s, then its values, beside which K of unit s + 2 is read.
    auto step = [&](int s, const floatx16 (&from)[R], floatx16 (&to)[R], bool masks) {  // from: the scores of unit s, to: those of unit s + 1
      ready();
      feed.next();
      score_half<D, false, R, F::kReq>(k, st, from, to, pw, lane_v + v_at, v, c2, [&](int i) { feed.request(i); });
      feed.requested(true, true);
      if (masks) mask(s + 1, to);
      add_half<D, false, R, true>(k, lane_k + k_at, lane_v + v_at, v, st, pw, to, mx, ones);
      check(mx);
      advance_k();
      advance_v();
    };
    int s = 0;
    for (; s + 2 < nst && !masked(s + 2); s += 2) {  // (the scores alternate between two sets of registers)
      step(s, sc, sd, false);
      step(s + 1, sd, sc, false);
    }
    for (; s + 1 < nst; s++) {
      step(s, sc, sd, true);
#pragma unroll
      for (int t = 0; t < R; t++) sc[t] = sd[t];
    }
    ready();
    bf16x8 pb[R][2];
#pragma unroll
    for (int t = 0; t < R; t++) {
      probs<D, false>(sc[t], st[t], c2, pb[t]);
#pragma unroll
      for (int j = 0; j < 2; j++) st[t].lacc = __builtin_amdgcn_mfma_f32_16x16x32_bf16(ones, pb[t][j], st[t].lacc, 0, 0, 0);
    }
#pragma unroll
    for (int j = 0; j < 2; j++)
#pragma unroll
      for (int dt = 0; dt < D / 32; dt++) {
        const bf16x8 a = read_v<D>(lane_v + v_at, dt, j);
#pragma unroll
        for (int t = 0; t < R; t++) st[t].o[dt] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(a, pb[t][j], st[t].o[dt], 0, 0, 0);
      }
  };
  auto careful_sweep = [&] {  // a unit at a time
    for (int s = 0; s < nst; s++) {
      wait_vmcnt<0>();
      ring_barrier();
      if (s > 0) feed.request_step();
      if (has_rows) {
        uint4 k[D / 16];
        floatx16 sc[R];
        bf16x8 pb[R][2];
        float mx[R];
        bool odd_v = false, odd_p = false;
        read_k<D>(lane_k + k_at, k);
        scores<D, R>(k, st, sc);
        mask(s, sc);
#pragma unroll
        for (int t = 0; t < R; t++) mx[t] = row_max(sc[t]);
        check(mx);
#pragma unroll
        for (int t = 0; t < R; t++) {
          probs<D, false>(sc[t], st[t], c2, pb[t]);
#pragma unroll
          for (int j = 0; j < 2; j++) st[t].lacc = __builtin_amdgcn_mfma_f32_16x16x32_bf16(ones, finite_only(pb[t][j], odd_p), st[t].lacc, 0, 0, 0);
        }
#pragma unroll
        for (int j = 0; j < 2; j++)
#pragma unroll
          for (int dt = 0; dt < D / 32; dt++) {
            const bf16x8 a = finite_only(read_v<D>(lane_v + v_at, dt, j), odd_v);
#pragma unroll
            for (int t = 0; t < R; t++) st[t].o[dt] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(a, pb[t][j], st[t].o[dt], 0, 0, 0);
          }
        if (__builtin_amdgcn_ballot_w64(odd_v) != 0)
#pragma unroll
          for (int t = 0; t < R; t++) add_odd_values<D>(st[t].o, pb[t][0], pb[t][1], vring + v_at, (seen[t] < k1 ? seen[t] : k1) - k0 - s * kUnitKeys, l);
      }
      advance_k();
      advance_v();
    }
  };
  if constexpr (CARE) careful_sweep();
  else if (has_rows) sweep();
  else {  // no rows of its own: it only brings its share, passing the same barriers
    for (int s = 0; s + 1 < nst; s++) {
      ready();
      feed.request_step();
      advance_v();
    }
    ready();
  }
  wait_vmcnt<0>();  // (the requests past the split's end, before the ring serves anything else)
  if (!CARE && any_odd<D>(st, sh.odd, w, l)) return true;
#pragma unroll
  for (int t = 0; t < R; t++) {
    floatx4 f[Part::P];
#pragma unroll
    for (int pc = 0; pc < Part::P; pc++) {
      const floatx16& o = st[t].o[pc >> 2];
      f[pc] = floatx4{o[4 * (pc & 3)], o[4 * (pc & 3) + 1], o[4 * (pc & 3) + 2], o[4 * (pc & 3) + 3]};
    }
    write_rows<D, 32, true, Part::P>(p, jb, w * R + t, grow[t], f, 0, st[t].mref, st[t].lacc[0], c2, true, l);
  }
  return false;
}

// The split merge by the last workgroup of a tile to arrive (split_merge's, for tiles whose row tiles are a wavefront's each): a wavefront
// has a row tile's whole states of two splits under way at once, where a few pieces at a time are a round trip to memory each (tiles of 128 rows
// in two splits: 8 us at the end of a workgroup).  The splits are added up in their order, whoever arrives last.
template <int D>
__device__ __forceinline__ void merge_by_last(const AttnParams& p, const TileJob& jb, int* flag_lds) {
  constexpr int P = PartialLayout<D, 32, true>::P;
  const int tid = threadIdx.x, w = __builtin_amdgcn_readfirstlane(tid >> 6), l = tid & 63;
  CB_GLOBAL unsigned long long* const ticket = (CB_GLOBAL unsigned long long*)p.tickets + 2 * (((int64_t)jb.b * p.Hkv + jb.hk) * jb.tiles + jb.rt);
  const unsigned long long xcc = __builtin_amdgcn_s_getreg(20 | (0 << 6) | ((4 - 1) << 11)) & 15u;
  asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
  __syncthreads();
  if (tid == 0) {
    const unsigned long long arrive = 1ull | (xcc << 24) | ((xcc * xcc) << 40);
    const unsigned long long tot = __hip_atomic_fetch_add(ticket, arrive, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT) + arrive, n = tot & 0xfffull;
    int flag = n == (unsigned long long)jb.nsplit ? 1 : 0;
    if (flag) {
      if (((tot >> 24) & 0xffffull) != n * xcc || tot >> 40 != n * xcc * xcc) flag = 2;  // (some split ran on another XCD: not in this L2)
      __hip_atomic_store(ticket, 0ull, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);      // ready for the next launch
    }
    *flag_lds = flag;
  }
  __syncthreads();
  const int flag = *flag_lds;
  if (!flag) return;
  const __amdgpu_buffer_rsrc_t prsrc = partial_rsrc<D, 32, true>(p, jb);
  const int rows = jb.M - jb.row0 < p.tile_rows ? jb.M - jb.row0 : p.tile_rows;
  for (int i = w; i * 32 < rows; i += kWideWaves) {
    const int row = jb.row0 + i * 32 + (l & 31), token = row / jb.g;
    const int64_t gr = row < jb.M ? (int64_t)(jb.off + token) * p.Hq + jb.hk * jb.g + (row - token * jb.g) : -1;
    const uint32_t byte = partial_byte<D, 32, true>(p, jb, i);
    if (flag == 1) merge_pieces<D, 32, true, P, 0, 2, true>(prsrc, gr, byte, (CB_GLOBAL uint16_t*)p.out, jb.nsplit, 0, l);
    else merge_pieces<D, 32, true, P, kAgentCoherent, 2, true>(prsrc, gr, byte, (CB_GLOBAL uint16_t*)p.out, jb.nsplit, 0, l);
  }
}

template <int D, bool PG>
__global__ __launch_bounds__(64 * kWideWaves, 1) void k_chunk_few(AttnParams p_arg, SeqMeta meta, ChunkSplits splits) {
  const SeqMetaLanes ml = seq_meta_prefetch(meta);
  const int lane_chunk = splits.keys[threadIdx.x & 63];
  __shared__ __align__(1024) uint4 ring[Feed<D, kWideWaves, 32>::kRingVecs];
  __shared__ TileLds sh;
  __shared__ int odd[kWideWaves];
  AttnParams p = p_arg;
  pin_args(p);
  TileJob jb;
  if (!chunk_job(p, ml, lane_chunk, blockIdx.x, jb)) return;
  if (sweep_few<D, PG, false>(p, jb, sh, odd, ring)) sweep_few<D, PG, true>(p, jb, sh, odd, ring);
  if (jb.nsplit > 1) split_merge<D, 32, true, kWideWaves, 128, false, true>(p, jb, p.tile_rows, sh, nullptr, [] {});
}

template <int D, bool PG>
__global__ __launch_bounds__(64 * kWideWaves, 1) void k_chunk_tall(AttnParams p_arg, SeqMeta meta, ChunkSplits splits) {
  const SeqMetaLanes ml = seq_meta_prefetch(meta);
  const int lane_chunk = splits.keys[threadIdx.x & 63];
  __shared__ __align__(1024) uint4 ring[Feed<D, kWideWaves, 32>::kRingVecs];
  __shared__ TileLds sh;
  __shared__ int odd[kWideWaves];
  AttnParams p = p_arg;
  pin_args(p);
  TileJob jb;
  if (!chunk_job(p, ml, lane_chunk, blockIdx.x, jb)) return;
  if (sweep_tall<D, PG, false>(p, jb, sh, odd, ring)) sweep_tall<D, PG, true>(p, jb, sh, odd, ring);
  if (jb.nsplit == 1) return;
  if (p.coop_merge) split_merge<D, 32, true, kWideWaves, 256, false, true>(p, jb, p.tile_rows, sh, nullptr, [] {});
  else merge_by_last<D>(p, jb, &sh.flag);
}

template <int D, bool PG>
__global__ __launch_bounds__(64 * kWideWaves, 2) void k_chunk_many(AttnParams p_arg, SeqMeta meta, ChunkSplits splits) {
  const SeqMetaLanes ml = seq_meta_prefetch(meta);
  const int lane_chunk = splits.keys[threadIdx.x & 63];
  __shared__ __align__(1024) ManyLds<D> sh;
  AttnParams p = p_arg;
  pin_args(p);
  TileJob jb;
  if (!chunk_job(p, ml, lane_chunk, blockIdx.x, jb)) return;
  if (sweep_many<D, PG, false>(p, jb, sh)) sweep_many<D, PG, true>(p, jb, sh);
  if (jb.nsplit == 1) return;
  if (!p.coop_merge) {
    merge_by_last<D>(p, jb, &sh.flag);
    return;
  }
  __syncthreads();  // (everybody is done with the rings, whose place the merge's words take)
  static_assert(sizeof(TileLds) <= sizeof(sh.ring), "");
  split_merge<D, 32, true, kWideWaves, 128, false, true>(p, jb, p.tile_rows, *reinterpret_cast<TileLds*>(sh.ring), nullptr, [] {});
}

int64_t chunk_partial_bytes(int D, int64_t total, int Hq, int Hkv, int batch) {
  const int64_t tiles = total * Hq / 32 + (int64_t)(Hkv + 1) * batch + 1;  // (block_tile0)
  return tiles * (D == 64 ? PartialLayout<64, 32, true>::kBytes : PartialLayout<128, 32, true>::kBytes);
}

template <int D>
static hipError_t launch_dim(hipStream_t st, const AttnParams& p, const SeqMeta& meta, const ChunkSplits& splits, int wgs) {
  const dim3 grid(wgs), block(64 * kWideWaves);
  const bool paged = p.kv.block_size > 0;
  if (p.tile_rows == 64 && paged) hipLaunchKernelGGL((k_chunk_few<D, true>), grid, block, 0, st, p, meta, splits);
  else if (p.tile_rows == 64) hipLaunchKernelGGL((k_chunk_few<D, false>), grid, block, 0, st, p, meta, splits);
  else if (p.tile_rows == 128 && paged) hipLaunchKernelGGL((k_chunk_many<D, true>), grid, block, 0, st, p, meta, splits);
  else if (p.tile_rows == 128) hipLaunchKernelGGL((k_chunk_many<D, false>), grid, block, 0, st, p, meta, splits);
  else if (D == 64) return hipErrorInvalidValue;  // (4096 tokens, 32/8 heads: 118 us, with tiles of 128 rows 97)
  else if (paged) hipLaunchKernelGGL((k_chunk_tall<128, true>), grid, block, 0, st, p, meta, splits);
  else hipLaunchKernelGGL((k_chunk_tall<128, false>), grid, block, 0, st, p, meta, splits);
  return hipGetLastError();
}
hipError_t launch_attn_chunk(hipStream_t st, const AttnParams& p, const SeqMeta& meta, const ChunkSplits& splits, int wgs) {
  return p.D == 64 ? launch_dim<64>(st, p, meta, splits, wgs) : launch_dim<128>(st, p, meta, splits, wgs);
}

}  // namespace cb
