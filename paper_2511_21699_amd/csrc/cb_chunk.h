// What the kernels of a chunk's attention share (cb_attn_chunk.hip, cb_attn_chunk_f32.hip).  gfx950 only.
#pragma once
#include "cb_attn_tile.h"

namespace cb {

// The workgroup's (tile, split); lane_chunk: lane b has sequence b's keys per split.  p.grid_x: workgroups.  They are numbered sequence by sequence, the longest first, a sequence's tiles from the last, whose
// sweep is the longest, to the first, then splits, and the kv head runs fastest: what is dispatched last is short, and with a
// multiple of 8 kv heads a head's tiles share an XCD's L2.
__device__ __forceinline__ bool chunk_job(const AttnParams& p, const SeqMetaLanes& ml, int lane_chunk, int d, TileJob& j) {
  // Two workgroups to a compute unit: numbers 256 to 511 go where 0 to 255 have gone, in that order, so they are taken from the shortest on, in
  // stretches of 8 that keep their XCD (a prompt of 2048, 32 heads: 64 stages and 1 on a compute unit instead of 64 and 32).
  if (d >= 256 && d < 512 && p.grid_x % 8 == 0) {
    const int end = p.grid_x < 512 ? p.grid_x : 512;
    d = 256 + end - 8 - (d & ~7) + (d & 7);
  }
  const int i = __popcll(__builtin_amdgcn_ballot_w64(ml.start <= d)) - 1;  // (starts past the batch are INT_MAX)
  j.b = __builtin_amdgcn_readlane(ml.ord, i);
  const int at = d - __builtin_amdgcn_readlane(ml.start, i);
  const SeqShape s = seq_shape(ml, j.b);
  j.g = p.Hq / p.Hkv;
  j.hk = at % p.Hkv;
  j.M = s.N * j.g;
  const int chunk = __builtin_amdgcn_readlane(lane_chunk, j.b), rest = at / p.Hkv, splits = (s.S + s.N + chunk - 1) / chunk, tiles = (j.M + p.tile_rows - 1) / p.tile_rows;
  j.split = rest % splits;
  j.rt = tiles - 1 - rest / splits;
  j.tiles = p.grid_y;
  j.off = s.off;
  j.N = s.N;
  j.S = s.S;
  j.layer = 0;
  j.row0 = j.rt * p.tile_rows;
  const int last = (j.row0 + p.tile_rows < j.M ? j.row0 + p.tile_rows : j.M) - 1, len = s.S + last / j.g + 1;
  j.k0 = j.split * chunk;
  if (j.k0 >= len) return false;
  j.k1 = j.k0 + chunk < len ? j.k0 + chunk : len;
  j.nsplit = (len + chunk - 1) / chunk;
  return true;
}

}  // namespace cb
