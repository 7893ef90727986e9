// What the kernels of a chunk's attention share (cb_attn_chunk.hip, cb_attn_chunk_f32.hip).  gfx950 only.
#pragma once
#include "cb_attn_tile.h"

namespace cb {

// The workgroup's (tile, split); lane_chunk: lane b has the most keys of a split of sequence b.  p.grid_x: workgroups.  They are numbered sequence by sequence, the longest
// first, a sequence's tiles from the last, whose sweep is the longest, to the first, then splits, and the kv head runs fastest: what is dispatched last is short, and with a
// multiple of 8 kv heads a head's tiles share an XCD's L2.
__device__ __forceinline__ bool chunk_job(const AttnParams& p, const SeqMetaLanes& ml, int lane_chunk, int d, TileJob& j) {
  // Two workgroups to a compute unit (tiles of 128 rows): numbers 256 to 511 go where 0 to 255 have gone, in that order, so they are taken from the shortest on, in
  // stretches of 8 that keep their XCD (a prompt of 2048, 32 heads: 64 stages and 1 on a compute unit instead of 64 and 32).
  // Where a compute unit has one workgroup at a time the next one dispatched is to be the longest left (fp32, 512 tokens, 32/8 heads: 45 us, and 53 that way).
  if (p.tile_rows == 128 && d >= 256 && d < 512 && p.grid_x % 8 == 0) {
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
  j.nsplit = (len + chunk - 1) / chunk;
  if (j.split >= j.nsplit) return false;
  const int part = ((len + j.nsplit - 1) / j.nsplit + 31) & ~31;  // (at most `chunk`: the tile's splits are of one length too)
  j.k0 = j.split * part;
  j.k1 = j.k0 + part < len ? j.k0 + part : len;
  return true;
}

}  // namespace cb
