// The plan of a batch of packed sequences, as the kernels read it.
//
// A plan holds, for packed_max_tiles() tiles of PACKED_ROWS rows at most, a
// PackedTile each, in order of falling work, then one int32 per row: its position
// in its sequence, or -1.  The lengths are known on the device only, so launches
// cover as many tiles as there can be; entries past the last tile have len 0.
#pragma once
#include "common.h"
#include "kernels.h"

namespace ls {

// Tile `rank` (0-based, rows PACKED_ROWS * rank .. of the sequence) of the sequence of
// `len` rows from row `start` on.  A query tile of rank r sees r + 1 tiles of
// keys; the key tile with r tiles of queries after it does the same work, so one
// list serves both: it is key tile (tiles of the sequence) - 1 - r.
struct PackedTile {
  int32_t start, len, rank, pad;
};

inline const PackedTile* packed_tiles(const void* plan) { return (const PackedTile*)plan; }
inline const int32_t* packed_pos(const PackedShape& p, const void* plan) {
  return (const int32_t*)((const char*)plan + packed_tile_bytes(p));
}

// Entry i of the list; len 0 where there is none.  Whatever a plan holds (lengths
// that were not in order, memory that was never filled), the entry returned lies
// inside the `total` rows, so that nothing outside a buffer is touched.
LS_DEV PackedTile packed_tile(const PackedTile* tiles, int i, int total) {
  PackedTile t = tiles[i];
  t.start = __builtin_amdgcn_readfirstlane(t.start);
  t.len = __builtin_amdgcn_readfirstlane(t.len);
  t.rank = __builtin_amdgcn_readfirstlane(t.rank);
  if (t.start < 0 || t.start >= total || t.len <= 0 || t.len > total - t.start || t.rank < 0 ||
      t.rank > (t.len - 1) / PACKED_ROWS)
    t = PackedTile{0, 0, 0, 0};
  return t;
}

}  // namespace ls
