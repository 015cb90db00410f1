"""The head loss without a GPU: what its calls refuse, and its workspace."""
from __future__ import annotations

import pytest
import torch

from paper_2510_02483_amd import lib as L

NULL, SHAPE, UNSUPPORTED, ALIGN, ALIAS, WORKSPACE = 1, 2, 3, 4, 5, 6
A = 1 << 30  # addresses are compared, never followed, by a call that refuses
DEFAULT = object()


def need(T=100, H=64, V=1003, piece=0):
    return L.lib().ls_head_loss_workspace(T, H, V, piece)


def fwd(T=100, H=64, V=1003, h=A, e=2 * A, t=3 * A, loss=4 * A, rows=5 * A, lse=6 * A, ws=7 * A, n=DEFAULT):
    return L.lib().ls_head_loss_fwd(T, H, V, h, e, t, loss, rows, lse, ws, need(T, H, V) if n is DEFAULT else n, None)


def bwd(T=100, H=64, V=1003, h=A, e=2 * A, t=3 * A, lse=4 * A, dloss=5 * A, dh=6 * A, de=7 * A, acc=0, low=None, piece=0,
        ws=8 * A, n=DEFAULT):
    return L.lib().ls_head_loss_bwd(T, H, V, h, e, t, lse, dloss, dh, de, acc, low, piece, ws,
                                    need(T, H, V, piece) if n is DEFAULT else n, None)


@pytest.mark.parametrize("call", [fwd, bwd])
@pytest.mark.parametrize("bad", [dict(T=0), dict(T=-1), dict(H=0), dict(H=60), dict(V=0), dict(V=1 << 30),
                                 dict(T=1 << 30, H=64), dict(T=1 << 24, H=64)])
def test_shapes_refused(call, bad):
    assert call(n=1 << 50, **bad) == SHAPE
    assert need(**bad) == 0


def test_forward_refusals():
    for name in ("h", "e", "t", "loss", "rows", "lse", "ws"):
        assert fwd(**{name: None}) == NULL, name
        assert fwd(**{name: A + 8 if name == "h" else 20 * A + 4}) == ALIGN, name
    assert fwd(lse=A) == ALIAS and fwd(rows=4 * A) == ALIAS and fwd(ws=2 * A) == ALIAS
    assert fwd(n=0) == WORKSPACE


def test_backward_refusals():
    for name in ("h", "e", "t", "lse", "ws"):
        assert bwd(**{name: None}) == NULL, name
    assert bwd(dh=None, de=None) == NULL
    assert bwd(low=9 * A) == UNSUPPORTED
    assert bwd(piece=-1, n=1 << 50) == SHAPE and need(piece=-1) == 0
    assert bwd(dh=A) == ALIAS and bwd(de=2 * A) == ALIAS and bwd(de=None, low=6 * A) == ALIAS and bwd(dh=5 * A) == ALIAS
    assert bwd(dh=6 * A + 2) == ALIGN and bwd(dloss=5 * A + 4) == ALIGN
    assert bwd(n=need() // 2) == WORKSPACE
    t = torch.zeros(1, dtype=torch.int32)
    with pytest.raises(ValueError):
        L.ls_head_loss_bwd(torch.zeros(1, 8), torch.zeros(3, 8), t, None, None, None,
                           torch.zeros(3, 8, dtype=torch.bfloat16), True, None)
    for bad in (t.long(), torch.zeros(2, dtype=torch.int32)):  # read as int32, one per row
        with pytest.raises(ValueError):
            L.ls_head_loss_fwd(torch.zeros(1, 8), torch.zeros(3, 8), bad, None, None, None, None)
        with pytest.raises(ValueError):
            L.ls_head_loss_bwd(torch.zeros(1, 8), torch.zeros(3, 8), bad, None, None, None, None, False, None)


def test_workspace_follows_the_piece():
    whole, small = need(4096, 1024, 100_000), need(4096, 1024, 100_000, 1024)
    # one piece of 64 columns' gradient is 2 bytes an entry; dh in fp32 beside it
    assert small < whole and small >= 4096 * 1024 * 2 + 4096 * 1024 * 4
    assert need(4096, 1024, 100_000, 1000) == small  # rounded up to a multiple of 64
    # never the logits: 4096 x 100000 x 2 bytes would be 781 MiB
    assert whole < 4096 * 100_000 * 2
    # head weights beyond what one operand of a product may be are taken in pieces
    assert need(256, 8192, 1_000_000) > 0


def test_workspace_does_not_depend_on_a_forced_tile():
    free = need(777, 512, 30_011)
    try:
        L.ls_gemm_tile_override(256, 192)
        assert need(777, 512, 30_011) == free
    finally:
        L.ls_gemm_tile_override(0, 0)
