"""Packed sequences without a GPU: what the calls refuse, the plan's size, and the
reference's gradients against differences."""
from __future__ import annotations

import ctypes

import numpy as np
import pytest
import torch

import packed_ref as R
from paper_2510_02483_amd import lib as L
from paper_2510_02483_amd.configs import PackedConfig

NULL, SHAPE, UNSUPPORTED, ALIGN, ALIAS, WORKSPACE = 1, 2, 3, 4, 5, 6
BASE = 1 << 20  # addresses are compared, never followed, by a call that refuses
BIG = 1 << 40


def cfg(total=300, n_seqs=3, nq=4, nkv=2, d=64):
    return L.LsPackedCfg(total, n_seqs, nq, nkv, d)


def plan(c, cu=BASE, p=BASE * 2, nbytes=BIG):
    return L.lib().ls_packed_plan(ctypes.byref(c), cu, p, nbytes, None)


def rope(c, p=BASE, nbytes=None, theta=1e4, src=BASE * 64, dst=BASE * 64):
    n = L.lib().ls_packed_plan_bytes(ctypes.byref(c)) if nbytes is None else nbytes
    return L.lib().ls_packed_rope(ctypes.byref(c), p, n, theta, 0, src, dst, None)


def fwd(c, p=BASE, nbytes=None, qkv=BASE * 64, o=BASE * 128, lse=BASE * 192):
    n = L.lib().ls_packed_plan_bytes(ctypes.byref(c)) if nbytes is None else nbytes
    return L.lib().ls_packed_attn_fwd(ctypes.byref(c), p, n, qkv, o, lse, None)


def bwd(c, p=BASE, nbytes=None, qkv=BASE * 64, o=BASE * 128, lse=BASE * 192, dout=BASE * 256, dqkv=BASE * 320,
        ws=BASE * 384, ws_bytes=None):
    n = L.lib().ls_packed_plan_bytes(ctypes.byref(c)) if nbytes is None else nbytes
    w = L.lib().ls_packed_attn_bwd_workspace(ctypes.byref(c)) if ws_bytes is None else ws_bytes
    return L.lib().ls_packed_attn_bwd(ctypes.byref(c), p, n, qkv, o, lse, dout, dqkv, ws, w, None)


CALLS = (plan, rope, fwd, bwd)


@pytest.mark.parametrize("call", CALLS)
@pytest.mark.parametrize("bad,status", [
    (dict(total=0), SHAPE), (dict(total=-5), SHAPE), (dict(n_seqs=0), SHAPE), (dict(nq=0), SHAPE), (dict(nkv=0), SHAPE),
    (dict(nq=3, nkv=2), SHAPE), (dict(d=100), UNSUPPORTED), (dict(d=32), UNSUPPORTED), (dict(d=136), UNSUPPORTED), (dict(d=0), SHAPE),
    (dict(total=1 << 28), SHAPE), (dict(n_seqs=1 << 28), SHAPE), (dict(total=(1 << 28) - 1, nq=16, nkv=8), SHAPE), (dict(nq=1 << 14, nkv=1), SHAPE),
])
def test_shapes_refused(call, bad, status):
    assert call(cfg(**bad), nbytes=BIG) == status
    assert L.lib().ls_last_error()


def test_null_alignment_alias_and_sizes():
    c = cfg()
    need = L.lib().ls_packed_plan_bytes(ctypes.byref(c))
    assert L.lib().ls_packed_plan(None, BASE, BASE, BIG, None) == NULL
    assert L.lib().ls_packed_rope(None, BASE, BIG, 1e4, 0, BASE, BASE, None) == NULL
    assert plan(c, cu=None) == NULL and plan(c, p=None) == NULL
    assert plan(c, cu=BASE + 4) == ALIGN and plan(c, p=2 * BASE + 8) == ALIGN
    assert plan(c, cu=BASE, p=BASE) == ALIAS
    assert plan(c, nbytes=need - 1) == WORKSPACE
    for call in (rope, fwd, bwd):
        assert call(c, p=None) == NULL and call(c, p=BASE + 2) == ALIGN
        assert call(c, nbytes=need - 1) == WORKSPACE
    assert rope(c, src=None) == NULL and rope(c, dst=None) == NULL
    assert rope(c, dst=BASE * 64 + 16) == ALIAS  # neither in place nor apart
    assert rope(c, p=BASE * 64) == ALIAS
    assert rope(c, theta=1.0) == SHAPE and rope(c, theta=float("nan")) == SHAPE and rope(c, theta=float("inf")) == SHAPE
    assert fwd(c, qkv=None) == NULL and fwd(c, o=None) == NULL and fwd(c, lse=None) == NULL
    assert fwd(c, o=BASE * 64) == ALIAS and fwd(c, lse=BASE * 128) == ALIAS and fwd(c, lse=BASE) == ALIAS
    assert bwd(c, dout=None) == NULL and bwd(c, ws=None) == NULL and bwd(c, dqkv=BASE * 64) == ALIAS
    assert bwd(c, ws_bytes=L.lib().ls_packed_attn_bwd_workspace(ctypes.byref(c)) - 1) == WORKSPACE
    assert bwd(c, dqkv=BASE * 320 + 8) == ALIGN


def test_lengths_of_another_type_or_number():
    """The library reads n_seqs + 1 int32; what torch makes of a cumulative sum is int64."""
    c = PackedConfig(300, 3, 4, 2, 64)
    buf = torch.zeros(1 << 16, dtype=torch.uint8)
    for bad in (torch.zeros(4, dtype=torch.int64), torch.zeros(3, dtype=torch.int32)):
        with pytest.raises(ValueError):
            L.ls_packed_plan(c, bad, buf)


def test_plan_has_room_for_every_batch_of_its_total():
    """16 bytes for each tile of up to 128 rows that any lengths can give, and 4 for each row."""
    rng = np.random.default_rng(0)
    for _ in range(200):
        n = int(rng.integers(1, 40))
        lens = rng.integers(0, rng.integers(1, 600) + 1, n)
        total = int(lens.sum()) + int(rng.integers(0, 50))
        if total == 0:
            continue
        tiles = int(((lens + 127) // 128).sum())
        c = cfg(total=total, n_seqs=n)
        assert L.lib().ls_packed_plan_bytes(ctypes.byref(c)) >= 16 * tiles + 4 * total
    assert L.lib().ls_packed_plan_bytes(ctypes.byref(cfg(d=56))) == 0
    assert L.lib().ls_packed_attn_bwd_workspace(ctypes.byref(cfg(total=0))) == 0


def test_reference_gradients_against_differences():
    rng = np.random.default_rng(1)
    lens, first, total, nq, nkv, d = [5, 0, 1, 9], 2, 20, 4, 2, 8
    x = rng.standard_normal((total, (nq + 2 * nkv) * d))
    do = rng.standard_normal((total, nq * d))
    do[:first] = do[first + sum(lens):] = 0.0
    grad = R.attention(x, lens, first, nq, nkv, d, do)[2]
    turned = R.rope(grad, lens, first, nq, nkv, d, 1e4, inverse=True)
    for g, f in ((grad, lambda y: y), (turned, lambda y: R.rope(y, lens, first, nq, nkv, d, 1e4))):
        if g is turned:  # the gradient at the rotation's input
            g = R.rope(R.attention(f(x), lens, first, nq, nkv, d, do)[2], lens, first, nq, nkv, d, 1e4, inverse=True)
        for _ in range(4):
            u = rng.standard_normal(x.shape)
            h = 1e-5
            up = (R.attention(f(x + h * u), lens, first, nq, nkv, d)[0] * do).sum()
            down = (R.attention(f(x - h * u), lens, first, nq, nkv, d)[0] * do).sum()
            # differences of order h^2 = 1e-10, cancellation 1e-16 * |L| / h = 1e-10
            assert abs((up - down) / (2 * h) - (g * u).sum()) < 1e-6 * (1 + abs((g * u).sum()))
