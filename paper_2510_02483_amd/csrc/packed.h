// The plan of a batch of packed sequences, as the kernels read it:
//   PackedHead, how many of the following there are;
//   PackedTile of every PACKED_ROWS rows of every sequence of more than PACKED_MID
//     rows, in order of falling work (and of the others, where they are few);
//   PackedTile (rank 0) of every middle sequence, of more than PACKED_SHORT and up to
//     PACKED_MID rows, and of every short one, of up to PACKED_SHORT;
//   PackedItem of every piece of work of the dK/dV kernel on tiles: a key tile, or
//     a part of the queries of one with many, in the tiles' order;
//   one int32 per row: its position in its sequence, or -1.
// The lengths are known on the device only, so the attention's launches cover as
// much work as there can be: unit u is tile u, or, past the tiles, middle and short
// sequences (four of them, one per wave, in the forward kernel; two middle ones,
// two waves each, or four short ones in the dK/dV kernel).
#pragma once
#include <algorithm>

#include "common.h"
#include "kernels.h"

namespace ls {

constexpr int PACKED_MID = 64;

struct PackedHead {
  int32_t tiles, mids, shorts, items, split;  // split: the first tiles, whose work is cut into parts
};

// Tile `rank` (0-based, rows PACKED_ROWS * rank .. of the sequence) of the sequence of
// `len` rows from row `start` on.  A query tile of rank r sees r + 1 tiles of
// keys; the key tile with r tiles of queries after it does the same work, so one
// list serves both: it is key tile (tiles of the sequence) - 1 - r.
// parts, slot: how many workgroups share the tile's dK/dV per kv head, and, when
// there are several, where their partial sums lie (slots slot .. slot + parts - 1).
struct PackedTile {
  int32_t start, len, rank;
  uint32_t parts : 10, slot : 22;
};
// A piece of dK/dV work: part `part` of a tile.
struct PackedItem {
  PackedTile tile;
  int32_t part, pad[3];
};

// Where the parts of a plan lie.
struct PackedLayout {
  int64_t max_tiles, max_mids, max_shorts, max_items, max_slots, max_units;
  size_t tiles, mids, shorts, items, pos, total;
};
// A key tile of rank r is r + 1 units of dK/dV work (128 queries) for every head of a kv
// head's group.  A tile with more than half of a compute unit's share of the tiles' work
// (in whole units of the group; less in small batches) is cut into parts of at most that.
// So there are at most 2 PACKED_CUS / nkv parts more than tiles, and as many tiles
// that are cut.
constexpr int PACKED_CUS = 256, PACKED_PART = 2;
// Middle and short sequences up to this many are listed as tiles where the heads of a group are many.
__host__ __device__ inline int packed_few(int nkv) { return PACKED_CUS / 4 / nkv; }
constexpr int PACKED_STEP = 64;  // queries of one head in a step of the dK/dV kernel
inline PackedLayout packed_layout(const PackedShape& p) {
  auto up = [](size_t x) { return (x + 255) & ~(size_t)255; };
  PackedLayout l;
  l.max_shorts = p.n_seqs < p.total ? p.n_seqs : p.total;
  // At most `big` sequences are long enough for tiles, and one of n rows has at most 1 + n / PACKED_ROWS.
  const int64_t big = std::min(l.max_shorts, p.total / (PACKED_MID + 1));
  l.max_tiles = std::max<int64_t>(big + p.total / PACKED_ROWS, 1);
  if (p.nq / p.nkv > PACKED_PART) l.max_tiles += std::min<int64_t>(l.max_shorts, packed_few(p.nkv));
  // The work that all sequences can make, in units: a sequence of tiles takes its tiles, a middle one half a unit and
  // more than half as many rows as the shortest of tiles, a short one a quarter.  So most units come from as many
  // sequences of tiles as the rows allow, and short ones for the rest.  (A workgroup without work costs about a
  // microsecond of its compute unit, which it must have to itself in the dK/dV kernel.)
  l.max_units = l.max_tiles + (l.max_shorts - big) / 4 + 2;
  const int64_t mids = (p.total + PACKED_SHORT) / (PACKED_SHORT + 1);
  l.max_mids = l.max_shorts < mids ? l.max_shorts : mids;
  l.tiles = 256;
  l.mids = l.tiles + up((size_t)l.max_tiles * sizeof(PackedTile));
  l.shorts = l.mids + up((size_t)l.max_mids * sizeof(PackedTile));
  l.max_items = l.max_tiles + 2 * PACKED_CUS / p.nkv;
  l.max_slots = 2 * (2 * PACKED_CUS / p.nkv);
  l.items = l.shorts + up((size_t)l.max_shorts * sizeof(PackedTile));
  l.pos = l.items + up((size_t)l.max_items * sizeof(PackedItem));
  l.total = l.pos + up((size_t)p.total * 4);
  return l;
}

// The plan as a kernel's argument.
struct PackedView {
  const PackedHead* head = nullptr;
  const PackedTile* tiles = nullptr;
  const PackedTile* mids = nullptr;
  const PackedTile* shorts = nullptr;
  const PackedItem* items = nullptr;
  int max_tiles = 0, max_mids = 0, max_shorts = 0, max_items = 0, max_slots = 0, max_units = 0;
};
inline PackedView packed_view(const PackedShape& p, const void* plan) {
  const PackedLayout l = packed_layout(p);
  const char* b = (const char*)plan;
  return PackedView{(const PackedHead*)b, (const PackedTile*)(b + l.tiles), (const PackedTile*)(b + l.mids),
                    (const PackedTile*)(b + l.shorts), (const PackedItem*)(b + l.items), (int)l.max_tiles,
                    (int)l.max_mids, (int)l.max_shorts, (int)l.max_items, (int)l.max_slots, (int)l.max_units};
}
// Tiles whose dK/dV work may be cut into parts (two slots each at least).
__host__ __device__ inline int packed_max_split(const PackedView& v) {
  return v.max_tiles < v.max_slots / 2 ? v.max_tiles : v.max_slots / 2;
}
inline const int32_t* packed_pos(const PackedShape& p, const void* plan) {
  return (const int32_t*)((const char*)plan + packed_layout(p).pos);
}

// A dimension of a launch holds fewer than 2^32 threads, which is 2^24 workgroups of 256: more lie in rows of
// PACKED_ROW_WGS, in the same order.  Those that the last row has too many find no work.
constexpr int PACKED_ROW_WGS = 1 << 23;
inline dim3 packed_grid(int64_t wgs) {
  if (wgs <= PACKED_ROW_WGS) return dim3((unsigned)wgs);
  return dim3(PACKED_ROW_WGS, (unsigned)((wgs + PACKED_ROW_WGS - 1) / PACKED_ROW_WGS));
}
LS_DEV int packed_wg() { return (int)(blockIdx.y * PACKED_ROW_WGS + blockIdx.x); }

// Whatever a plan holds (memory that was never filled, another shape's plan), the counts and entries returned lie inside the plan and the `total`
// rows, so that nothing outside a buffer is touched.  All uniform over a wave.
LS_DEV int packed_count(int n, int most) { return max(0, min(most, __builtin_amdgcn_readfirstlane(n))); }
LS_DEV PackedTile packed_checked(PackedTile t, int total) {
  t.start = __builtin_amdgcn_readfirstlane(t.start);
  t.len = __builtin_amdgcn_readfirstlane(t.len);
  t.rank = __builtin_amdgcn_readfirstlane(t.rank);
  if (t.start < 0 || t.start >= total || t.len <= 0 || t.len > total - t.start || t.rank < 0 ||
      t.rank > (t.len - 1) / PACKED_ROWS)
    t = PackedTile{};
  return t;
}
// Unit u of the forward and dQ kernels: tile u (true), or this wave's sequence of
// the four that unit u holds, middle ones first (false); len 0 where there is none.
// Counts and entry are loaded at once, not one after the other.
LS_DEV bool packed_unit(const PackedView& v, int u, int total, PackedTile& t) {
  const PackedHead h = *v.head;
  const PackedTile a = v.tiles[min(u, v.max_tiles - 1)];
  const int tiles = packed_count(h.tiles, v.max_tiles);
  if (u < tiles) {
    t = packed_checked(a, total);
    return true;
  }
  int i = __builtin_amdgcn_readfirstlane(4 * (u - tiles) + ((int)threadIdx.x >> 6));
  const int mids = packed_count(h.mids, v.max_mids);
  t = PackedTile{};
  if (i < mids) t = packed_checked(v.mids[i], total);
  else if ((i -= mids) < packed_count(h.shorts, v.max_shorts)) t = packed_checked(v.shorts[i], total);
  if (t.len > PACKED_MID) t = PackedTile{};
  return false;
}
// Unit u of the dK/dV kernel: a piece of the tiles' work, two middle sequences (this
// wave's: that of its pair) or four short ones.
enum PackedKind { PACKED_IS_TILE, PACKED_IS_MID, PACKED_IS_SHORT };
LS_DEV PackedKind packed_piece(const PackedView& v, int u, int total, PackedTile& t, int& part) {
  const PackedHead h = *v.head;
  const PackedItem a = v.items[min(u, v.max_items - 1)];
  const int items = packed_count(h.items, v.max_items);
  if (u < items) {
    t = packed_checked(a.tile, total);
    part = __builtin_amdgcn_readfirstlane(a.part);
    if (part < 0 || part >= (int)t.parts || (t.parts > 1 && (int)(t.slot + t.parts) > v.max_slots)) t = PackedTile{};
    return PACKED_IS_TILE;
  }
  u -= items;
  const int wave = __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6);
  const int mids = packed_count(h.mids, v.max_mids), units = (mids + 1) / 2;
  t = PackedTile{};
  if (u < units) {
    const int i = 2 * u + (wave >> 1);
    if (i < mids) t = packed_checked(v.mids[i], total);
    if (t.len > PACKED_MID) t = PackedTile{};
    return PACKED_IS_MID;
  }
  const int i = 4 * (u - units) + wave;
  if (i >= 0 && i < packed_count(h.shorts, v.max_shorts)) t = packed_checked(v.shorts[i], total);
  if (t.len > PACKED_SHORT) t = PackedTile{};
  return PACKED_IS_SHORT;
}

}  // namespace ls
