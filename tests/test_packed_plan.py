"""The lists of a plan and the launches over it have room for whatever lengths a total and a number of sequences allow."""
from __future__ import annotations

import ctypes
import random

import numpy as np
import pytest
import torch

import packed_ref as R
import plan_model as M
from paper_2510_02483_amd import lib as L
from paper_2510_02483_amd.configs import PackedConfig

HEADS = [(1, 1), (4, 2), (3, 1), (24, 8), (32, 2), (64, 1), (16, 16), (128, 32), (640, 64), (300, 300), (256, 128), (520, 520)]


def held(lens, total, nq, nkv):
    r, t = M.room(total, len(lens), nq, nkv, 64), M.taken(lens, total, nq, nkv)
    assert t.tiles <= r.tiles and t.mids <= r.mids and t.shorts <= r.shorts
    assert t.items <= r.items and t.slots <= r.slots
    assert t.split <= min(r.tiles, r.slots // 2)  # tiles that the joining workgroups cover
    assert t.forward_units() <= r.units and t.dkdv_units() <= r.units + r.items - r.tiles
    assert t.most_parts < 1 << 10 and r.slots < 1 << 22  # bits of a tile's entry
    return r, t


@pytest.mark.parametrize("nq,nkv", HEADS)
@pytest.mark.parametrize("d", [64, 72, 128])
def test_the_model_is_the_library(nq, nkv, d):
    rng = random.Random(1)
    for _ in range(60):
        total, n = rng.randrange(1, 1 << rng.randrange(1, 22)), rng.randrange(1, 1 << rng.randrange(1, 22))
        r = M.room(total, n, nq, nkv, d)
        c = L.LsPackedCfg(total, n, nq, nkv, d)
        assert L.lib().ls_packed_plan_bytes(ctypes.byref(c)) == r.plan_bytes
        assert L.lib().ls_packed_attn_bwd_workspace(ctypes.byref(c)) == r.work_bytes


@pytest.mark.parametrize("nq,nkv", HEADS)
def test_repeated_lengths_fill_the_room(nq, nkv):
    """Rows full of one length around the borders of the classes, or of two, with nothing left over or a few rows."""
    border = (1, 2, 32, 33, 64, 65, 66, 127, 128, 129, 192, 193, 256, 257, 640)
    for a in border:
        for k in (1, 2, 3, 5, 8, 63, 64, 65, 130):
            for b in (0,) + border:
                for j in (1, 4):
                    lens = [a] * k + ([b] * j if b else [])
                    for tail in (0, 1, 64):
                        held(lens, sum(lens) + tail, nq, nkv)


@pytest.mark.parametrize("nq,nkv", HEADS)
def test_random_lengths_fit_the_room(nq, nkv):
    rng = random.Random(nq * 1000 + nkv)
    for _ in range(400):
        top = rng.choice([1, 32, 64, 65, 130, 1000, 20_000])
        lens = [rng.choice([0, 1, 33, 65, 129, rng.randrange(0, top + 1)]) for _ in range(rng.randrange(1, 80))]
        if sum(lens):
            held(lens, sum(lens) + rng.choice([0, 0, 1, 200]), nq, nkv)


@pytest.mark.parametrize("nq,nkv", [(1, 1), (2, 1), (7, 1), (3, 3)])
def test_several_ranks_to_a_class(nq, nkv):
    rng = random.Random(5)
    for total in (300_000, 3_000_000, 50_000_000):
        for _ in range(12):
            lens, left = [], total
            while left > 0 and len(lens) < 60:
                lens.append(min(left, rng.choice([1, 65, 130, 5000, total // 3, total])))
                left -= lens[-1]
            held(lens, total, nq, nkv)


@pytest.mark.gpu
@pytest.mark.parametrize("nq,nkv", [(1, 1), (4, 2), (24, 8), (32, 2), (16, 16)])
def test_the_plan_holds_what_the_model_says(nq, nkv):
    """The counts at the plan's head: tiles, sequences of 33 to 64 and of up to 32 rows, pieces of dK/dV work, tiles cut."""
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    rng = np.random.default_rng(nq)
    mixes = [([5], 5), ([64, 33, 1, 0], 100), ([2500, 40, 3, 100], 2700), ([1] * 70, 70), ([130, 65, 300, 1], 3_000_000),
             ([33] * 40 + [17] * 40 + [700], 2800), ([4272, 2000, 900, 500, 200, 100, 100, 63], 8192)]
    mixes += [((x := rng.integers(0, 900, 30)).tolist(), int(x.sum()) + 7) for _ in range(3)]
    for lens, total in mixes:
        if total * nq >= 1 << 31:
            continue
        c = PackedConfig(total, len(lens), nq, nkv, 64)
        plan = torch.zeros(L.ls_packed_plan_bytes(c), dtype=torch.uint8, device="cuda")
        L.ls_packed_plan(c, torch.tensor(R.bounds_of(lens), dtype=torch.int32, device="cuda"), plan)
        t = M.taken(lens, total, nq, nkv)
        assert plan[:20].view(torch.int32).tolist() == [t.tiles, t.mids, t.shorts, t.items, t.split], (lens, total)
