"""The plan of a batch of packed sequences in plain Python: the room that its lists get from total and the number of
sequences, and how much of it lengths take."""
from __future__ import annotations

from collections import Counter
from dataclasses import dataclass

ROWS, MID, SHORT, CUS, PART, STEP, LEVELS = 128, 64, 32, 256, 2, 64, 2048


@dataclass
class Room:
    tiles: int
    mids: int
    shorts: int
    items: int
    slots: int
    units: int
    plan_bytes: int
    work_bytes: int  # of the backward's workspace


def room(total, n_seqs, nq, nkv, d):
    shorts = min(n_seqs, total)
    big = min(shorts, total // (MID + 1))
    tiles = max(big + total // ROWS, 1)
    if nq // nkv > PART:
        tiles += min(shorts, CUS // 4 // nkv)
    units = tiles + (shorts - big) // 4 + 2
    mids = min(shorts, -(-total // (SHORT + 1)))
    items, slots = tiles + 2 * CUS // nkv, 2 * (2 * CUS // nkv)

    def up(x):
        return -(-x // 256) * 256

    nbytes = 256 + up(16 * tiles) + up(16 * mids) + up(16 * shorts) + up(32 * items) + up(4 * total)
    work = up(8 * total * nq) + slots * nkv * ROWS * 2 * (64 if d == 64 else 128) * 4
    return Room(tiles, mids, shorts, items, slots, units, nbytes, work)


@dataclass
class Taken:
    tiles: int
    mids: int
    shorts: int
    items: int
    split: int
    slots: int
    most_parts: int

    def forward_units(self):
        return self.tiles + -(-(self.mids + self.shorts) // 4)

    def dkdv_units(self):
        return self.items + -(-self.mids // 2) + -(-self.shorts // 4)


def taken(lens, total, nq, nkv):
    group = nq // nkv
    shift = 0
    while ((total - 1) // ROWS) >> shift >= LEVELS:
        shift += 1
    classes = Counter()
    for n in lens:
        if n > MID:
            m = -(-n // ROWS)
            for c in range(((m - 1) >> shift) + 1):
                classes[c] += min(m - (c << shift), 1 << shift)
    mids, shorts = sum(SHORT < n <= MID for n in lens), sum(0 < n <= SHORT for n in lens)
    few, tiles = mids + shorts, sum(classes.values())

    def units(c):
        return ((c + 1) << shift) * group

    listed = group > PART and few <= CUS // 4 // nkv and tiles + few <= room(total, len(lens), nq, nkv, 64).tiles
    if listed:
        classes[0] += few
        tiles, mids, shorts = tiles + few, 0, 0
    work = sum(k * units(c) for c, k in classes.items())
    big = 1 << 30

    def share(w, n):
        return max(min(-(-w * nkv // n), big), PART)

    target = min(-(-share(work, 2 * CUS) // group) * group, share(work + (0 if listed else few * group), 64))
    parts = {c: min(-(-min(units(c), big) // target), 1023) for c in classes if classes[c]}
    cut = {c: p for c, p in parts.items() if p > 1}
    return Taken(tiles, mids, shorts, sum(classes[c] * p for c, p in parts.items()), sum(classes[c] for c in cut),
                 sum(classes[c] * p for c, p in cut.items()), max(parts.values(), default=0))
