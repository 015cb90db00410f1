"""Log probabilities of given tokens without a GPU: what the calls refuse, and their workspace."""
from __future__ import annotations

import pytest
import torch

from paper_2510_02483_amd import lib as L

NULL, SHAPE, UNSUPPORTED, ALIGN, ALIAS, WORKSPACE = 1, 2, 3, 4, 5, 6
A = 1 << 30  # addresses are compared, never followed, by a call that refuses
DEFAULT = object()


def need(T=100, H=64, V=1003, top=0, piece=0):
    return L.lib().ls_token_logprob_workspace(T, H, V, top, piece)


def fwd(T=100, H=64, V=1003, scale=1.0, h=A, e=2 * A, t=3 * A, logprob=4 * A, entropy=5 * A, lse=6 * A, top=5, ids=7 * A,
        vals=8 * A, ws=9 * A, n=DEFAULT):
    return L.lib().ls_token_logprob_fwd(T, H, V, scale, h, e, t, logprob, entropy, lse, top, ids, vals, ws,
                                        need(T, H, V, top) if n is DEFAULT else n, None)


def bwd(T=100, H=64, V=1003, scale=1.0, h=A, e=2 * A, t=3 * A, entropy=4 * A, lse=5 * A, dlogprob=6 * A, dentropy=7 * A,
        dh=8 * A, de=9 * A, acc=0, low=None, piece=0, ws=10 * A, n=DEFAULT):
    return L.lib().ls_token_logprob_bwd(T, H, V, scale, h, e, t, entropy, lse, dlogprob, dentropy, dh, de, acc, low, piece,
                                        ws, need(T, H, V, 0, piece) if n is DEFAULT else n, None)


@pytest.mark.parametrize("call", [fwd, bwd])
@pytest.mark.parametrize("bad", [dict(T=0), dict(T=-1), dict(H=0), dict(H=60), dict(V=0), dict(V=1 << 30),
                                 dict(T=1 << 30, H=64), dict(T=1 << 24, H=64)])
def test_shapes_refused(call, bad):
    assert call(n=1 << 50, **bad) == SHAPE
    assert need(**bad) == 0


@pytest.mark.parametrize("call", [fwd, bwd])
@pytest.mark.parametrize("scale", [0.0, -1.0, float("nan"), float("inf")])
def test_scales_refused(call, scale):
    assert call(scale=scale) == SHAPE


def test_forward_refusals():
    for name in ("h", "e", "t", "logprob", "entropy", "lse", "ids", "vals", "ws"):
        assert fwd(**{name: None}) == NULL, name
        assert fwd(**{name: 20 * A + 4}) == ALIGN, name
    assert fwd(top=-1, n=1 << 50) == SHAPE and fwd(top=65, n=1 << 50) == UNSUPPORTED
    assert need(top=-1) == 0 and need(top=65) == 0 and need(top=64) > 0
    assert fwd(lse=A) == ALIAS and fwd(entropy=4 * A) == ALIAS and fwd(ws=2 * A) == ALIAS and fwd(ids=8 * A) == ALIAS
    assert fwd(ids=3 * A) == ALIAS
    assert fwd(n=0) == WORKSPACE and fwd(n=4096) == WORKSPACE


def test_backward_refusals():
    for name in ("h", "e", "t", "entropy", "lse", "ws"):
        assert bwd(**{name: None}) == NULL, name
    assert bwd(dh=None, de=None) == NULL and bwd(dlogprob=None, dentropy=None) == NULL
    assert bwd(low=11 * A) == UNSUPPORTED and bwd(de=None, low=11 * A, acc=1) == UNSUPPORTED
    assert bwd(piece=-1, n=1 << 50) == SHAPE and need(piece=-1) == 0
    for out in ("dh", "de", "ws"):
        for at in (1, 2, 3, 4, 5, 6, 7):
            assert bwd(**{out: at * A}) == ALIAS, (out, at)
    assert bwd(dh=9 * A) == ALIAS and bwd(dh=8 * A + 2) == ALIGN and bwd(dlogprob=6 * A + 4) == ALIGN
    assert bwd(n=need() // 2) == WORKSPACE


def test_binding():
    T, H, V, k = 4, 8, 30, 3
    f32, i32, bf = torch.float32, torch.int32, torch.bfloat16
    spec = dict(h=(T, H, bf), embed=(V, H, bf), targets=(T, i32), logprob=(T, f32), entropy=(T, f32), lse=(T, f32),
                workspace=(64, torch.uint8), top_ids=(T, k, i32), top_logprob=(T, k, f32))
    good = {n: torch.zeros(*s, dtype=d) for n, (*s, d) in spec.items()}

    def bad(call, good, **other):
        with pytest.raises(ValueError):
            call(**dict(good, **other))

    f = L.ls_token_logprob_fwd
    for n in good:
        if n != "workspace":
            bad(f, good, **{n: good[n].double()})
        if n not in ("h", "embed"):
            bad(f, good, **{n: torch.cat([good[n], good[n]], -1)[..., ::2]})
    bad(f, good, targets=torch.zeros(T + 1, dtype=i32))
    bad(f, good, top_ids=None)
    bad(f, good, top_logprob=None)
    bad(f, good, top_logprob=torch.zeros(T, k - 1))
    bad(f, good, top_ids=torch.zeros(T, 0, dtype=i32), top_logprob=torch.zeros(T, 0))
    bad(f, good)  # host memory
    b = L.ls_token_logprob_bwd
    back = dict({n: good[n] for n in ("h", "embed", "targets", "entropy", "lse", "workspace")}, dlogprob=torch.zeros(T),
                dentropy=torch.zeros(T), dh=torch.zeros(T, H, dtype=bf), d_embed=torch.zeros(V, H), accumulate=False)
    bad(b, back)
    for n in ("dlogprob", "dentropy", "entropy", "lse"):
        bad(b, back, **{n: torch.zeros(T - 1)})
        bad(b, back, **{n: torch.zeros(T, dtype=bf)})
    bad(b, back, dh=torch.zeros(T, H))
    bad(b, back, d_embed=torch.zeros(V, H, dtype=bf), accumulate=True)


def test_workspace():
    whole, small = need(4096, 1024, 100_000), need(4096, 1024, 100_000, 0, 1024)
    assert small < whole < 4096 * 100_000 * 2  # never the logits
    # beside the plain one: 4 bytes for 16 logits, which the forward call alone needs
    assert need(4096, 1024, 100_000, 5) >= 4096 * 100_000 // 16 * 4
    assert need(4096, 1024, 100_000, 5) == need(4096, 1024, 100_000, 64)
    free = need(777, 512, 30_011, 5)
    try:
        L.ls_gemm_tile_override(256, 192)
        assert need(777, 512, 30_011, 5) == free
    finally:
        L.ls_gemm_tile_override(0, 0)
