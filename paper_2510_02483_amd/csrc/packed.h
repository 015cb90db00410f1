// The plan of a batch of packed sequences, as the kernels read it:
//   PackedHead, how many tiles and short sequences there are;
//   PackedTile of every PACKED_ROWS rows of every sequence that is not short, in
//     order of falling work, packed_max_tiles() of them at most;
//   PackedTile (rank 0) of every short sequence, of up to PACKED_SHORT rows;
//   one int32 per row: its position in its sequence, or -1.
// The lengths are known on the device only, so the attention's launches cover as
// many units of work as there can be: unit u is tile u, or, past the tiles, four short
// sequences, one per wave.
#pragma once
#include "common.h"
#include "kernels.h"

namespace ls {

struct PackedHead {
  int32_t tiles, shorts;
};

// Tile `rank` (0-based, rows PACKED_ROWS * rank .. of the sequence) of the sequence of
// `len` rows from row `start` on.  A query tile of rank r sees r + 1 tiles of
// keys; the key tile with r tiles of queries after it does the same work, so one
// list serves both: it is key tile (tiles of the sequence) - 1 - r.
struct PackedTile {
  int32_t start, len, rank, pad;
};

// Where the parts of a plan lie.
struct PackedLayout {
  int64_t max_tiles, max_shorts;
  size_t tiles, shorts, pos, total;
};
inline PackedLayout packed_layout(const PackedShape& p) {
  auto up = [](size_t x) { return (x + 255) & ~(size_t)255; };
  PackedLayout l;
  l.max_shorts = p.n_seqs < p.total ? p.n_seqs : p.total;
  // a sequence of n rows has at most (n + PACKED_ROWS - 1) / PACKED_ROWS tiles
  l.max_tiles = (p.total + (PACKED_ROWS - 1) * l.max_shorts) / PACKED_ROWS;
  l.tiles = 256;
  l.shorts = l.tiles + up((size_t)l.max_tiles * sizeof(PackedTile));
  l.pos = l.shorts + up((size_t)l.max_shorts * sizeof(PackedTile));
  l.total = l.pos + up((size_t)p.total * 4);
  return l;
}

// The plan as a kernel's argument.
struct PackedView {
  const PackedHead* head = nullptr;
  const PackedTile* tiles = nullptr;
  const PackedTile* shorts = nullptr;
  const int32_t* pos = nullptr;
  int max_tiles = 0, max_shorts = 0;
};
inline PackedView packed_view(const PackedShape& p, const void* plan) {
  const PackedLayout l = packed_layout(p);
  const char* b = (const char*)plan;
  return PackedView{(const PackedHead*)b, (const PackedTile*)(b + l.tiles), (const PackedTile*)(b + l.shorts),
                    (const int32_t*)(b + l.pos), (int)l.max_tiles, (int)l.max_shorts};
}

// Whatever a plan holds (lengths that were not in order, memory that was never
// filled), the counts and entries returned lie inside the plan and the `total`
// rows, so that nothing outside a buffer is touched.  All uniform over a wave.
LS_DEV int packed_tiles(const PackedView& v) {
  return max(0, min(v.max_tiles, __builtin_amdgcn_readfirstlane(v.head->tiles)));
}
LS_DEV PackedTile packed_entry(const PackedTile* list, int i, int total) {
  PackedTile t = list[i];
  t.start = __builtin_amdgcn_readfirstlane(t.start);
  t.len = __builtin_amdgcn_readfirstlane(t.len);
  t.rank = __builtin_amdgcn_readfirstlane(t.rank);
  if (t.start < 0 || t.start >= total || t.len <= 0 || t.len > total - t.start || t.rank < 0 ||
      t.rank > (t.len - 1) / PACKED_ROWS)
    t = PackedTile{0, 0, 0, 0};
  return t;
}
// Short sequence of `wave` (0..3) of unit u >= tiles; len 0 where there is none.
LS_DEV PackedTile packed_short(const PackedView& v, int unit, int tiles, int wave, int total) {
  const int i = __builtin_amdgcn_readfirstlane(4 * (unit - tiles) + wave);
  if (i >= min(v.max_shorts, __builtin_amdgcn_readfirstlane(v.head->shorts))) return PackedTile{0, 0, 0, 0};
  const PackedTile t = packed_entry(v.shorts, i, total);
  return t.len > PACKED_SHORT ? PackedTile{0, 0, 0, 0} : t;
}

}  // namespace ls
