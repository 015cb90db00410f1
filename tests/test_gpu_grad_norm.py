"""The norm of many gradient tensors and clipping by it, against 64 bits."""
from __future__ import annotations

import math

import numpy as np
import pytest
import torch

from gpu_util import need_gpu
from paper_2510_02483_amd import configs, inputs, lib as L

pytestmark = pytest.mark.gpu
BF16, F32 = torch.bfloat16, torch.float32


def make(sizes, types=(F32,), seed=0):
    g = torch.Generator().manual_seed(seed)
    return [(torch.randn(n, generator=g) * 10.0 ** -(i % 4)).to(types[i % len(types)]).cuda() for i, n in enumerate(sizes)]


def norm_of(ts, stream=None):
    out = torch.full((1,), -1.0, device="cuda")
    ws = torch.empty(L.ls_grad_norm_workspace(), dtype=torch.uint8, device="cuda")
    L.ls_grad_norm(ts, out, ws, stream=stream)
    return out


def want_norm(ts):
    return math.sqrt(sum(float((t.double() ** 2).sum()) for t in ts))


def factor(norm, max_norm):
    """The library's factor from its own norm: a quotient in 64 bits, rounded to 32."""
    return np.float32(min(1.0, float(np.float32(max_norm)) / (norm.item() + 1e-6)))


SIZES = {
    "one": [1],
    "few": [7, 0, 16384, 16385, 8, 1000],
    "odd": [3, 5, 16383, 4097, 12],
    "empty": [0, 0],
    "many": [1 + 37 * i % 500 for i in range(300)],
    "empty_many": [0] * 200 + [5] + [0] * 200,
    "large": [5_000_001, 33, 40_000_000],
    "two_tables": [20_000] * 97,
}


@pytest.mark.parametrize("types", [(F32,), (BF16,), (F32, BF16, BF16)], ids=["fp32", "bf16", "mixed"])
@pytest.mark.parametrize("sizes", SIZES, ids=list(SIZES))
def test_norm_and_clip(sizes, types):
    need_gpu()
    ts = make(SIZES[sizes], types)
    norm, ref = norm_of(ts), want_norm(ts)
    assert abs(norm.item() - ref) <= 2.0 ** -24 * ref * 1.01  # one rounding
    for max_norm in (0.5 * ref + 1e-3, 2.0 * ref + 1.0):
        f = torch.tensor(factor(norm, max_norm), device="cuda")
        for out_type in (None, F32, BF16):
            want = [(t.float() * f).to(out_type or t.dtype) for t in ts]
            if out_type is None:
                out = [t.clone() for t in ts]
                L.ls_grad_clip(out, norm, max_norm)
            else:
                out = [torch.full(t.shape, 7.0, dtype=out_type, device="cuda") for t in ts]
                L.ls_grad_clip(ts, norm, max_norm, out)
            assert all(torch.equal(a, b) for a, b in zip(out, want)), (max_norm, out_type)


def test_neighbours_of_a_tensor_stay():
    """Tensors inside an arena, 16 bytes apart: nothing between them is written."""
    need_gpu()
    arena = torch.ones(4000, device="cuda")
    views = [arena[0:5], arena[8:1001], arena[1004:1004], arena[1008:3999]]
    norm = norm_of(views)
    L.ls_grad_clip(views, norm, 1.0)
    left = torch.ones(4000, dtype=torch.bool, device="cuda")
    for a, b in ((0, 5), (8, 1001), (1008, 3999)):
        left[a:b] = False
    assert (arena[left] == 1.0).all() and (arena[~left] < 1.0).all()


def test_some_in_place_some_elsewhere():
    need_gpu()
    ts = make([100, 30, 1000])
    norm = norm_of(ts)
    f = torch.tensor(factor(norm, 0.1), device="cuda")
    want = [t * f for t in ts]
    out = [ts[0], torch.zeros_like(ts[1]), ts[2]]
    keep = ts[1].clone()
    L.ls_grad_clip(ts, norm, 0.1, out)
    assert all(torch.equal(a, b) for a, b in zip(out, want)) and torch.equal(ts[1], keep)


def test_values_whose_squares_overflow_or_vanish():
    need_gpu()
    for x in (1e30, 1e-30):
        ts = [torch.full((1000,), x, device="cuda"), torch.full((24,), x, device="cuda").to(BF16)]
        ref = want_norm(ts)
        assert abs(norm_of(ts).item() - ref) <= 2.0 ** -23 * ref


def test_infinite_and_nan_gradients():
    need_gpu()
    a, b = make([1000, 2000])
    b[77] = float("inf")
    norm = norm_of([a, b])
    assert torch.isinf(norm).all()
    out = [torch.ones_like(a), torch.ones_like(b)]
    L.ls_grad_clip([a, b], norm, 1.0, out)
    assert not out[0].any() and torch.isnan(out[1][77]) and not out[1][:77].any()
    b[77] = float("nan")
    norm = norm_of([a, b])
    assert torch.isnan(norm).all()
    L.ls_grad_clip([a, b], norm, 1.0, out)
    assert torch.isnan(out[0]).all() and torch.isnan(out[1]).all()


def test_the_same_tensor_twice_counts_twice():
    need_gpu()
    (a,) = make([777])
    assert abs(norm_of([a, a]).item() - math.sqrt(2.0) * want_norm([a])) < 1e-5
    with pytest.raises(L.LsError):  # but is not clipped twice
        L.ls_grad_clip([a, a], norm_of([a]), 1.0)


def test_replays_and_another_stream():
    need_gpu()
    ts = make([100_000, 3, 70_000], (F32, BF16))
    norm, ws = torch.zeros(1, device="cuda"), torch.empty(L.ls_grad_norm_workspace(), dtype=torch.uint8, device="cuda")
    out = [torch.zeros_like(t) for t in ts]
    g = torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    with torch.cuda.graph(g):
        L.ls_grad_norm(ts, norm, ws)
        L.ls_grad_clip(ts, norm, 0.25, out)
    for k in range(3):
        for t, new in zip(ts, make([100_000, 3, 70_000], (F32, BF16), seed=k + 1)):
            t.copy_(new)
        eager = norm_of(ts)
        want = [torch.zeros_like(t) for t in ts]
        L.ls_grad_clip(ts, eager, 0.25, want)
        torch.cuda.synchronize()
        g.replay()
        torch.cuda.synchronize()
        assert torch.equal(norm, eager) and all(torch.equal(a, b) for a, b in zip(out, want))
    s = torch.cuda.Stream()
    torch.cuda.synchronize()
    other = norm_of(ts, stream=s)
    s.synchronize()
    assert torch.equal(other, eager)


def test_a_block_step_clipped_and_stepped():
    """The block's nine gradients, clipped together, then AdamW tensor by tensor: what one flat array gives."""
    need_gpu()
    c = configs.TINY
    blk = L.Block(c, inputs.make_inputs(c, gamma="random"))
    blk.step()
    names = list(L.WEIGHTS)
    grads = [blk.grads[n] for n in names]
    norm = norm_of(grads)
    flat = torch.cat([g.reshape(-1) for g in grads])
    kw = dict(step=1, lr=1e-3, weight_decay=0.0)
    master = torch.cat([blk.w[n].float().reshape(-1) for n in names])
    m, v, one = torch.zeros_like(master), torch.zeros_like(master), torch.zeros(1, device="cuda")
    start = master.clone()
    L.ls_adamw_step(master, None, flat, m, v, max_norm=0.5 * norm.item(), grad_norm=one, **kw)
    assert abs(one.item() - norm.item()) <= 2.0 ** -23 * norm.item()
    L.ls_grad_clip(grads, norm, 0.5 * norm.item())
    at = 0
    for n, g in zip(names, grads):
        part = slice(at, at + g.numel())
        p, pm, pv = start[part].clone(), torch.zeros_like(m[part]), torch.zeros_like(v[part])
        L.ls_adamw_step(p, None, g.reshape(-1), pm, pv, max_norm=None, **kw)
        # (the factor comes from the rounded norm here)
        assert torch.allclose(pm, m[part], rtol=1e-5, atol=0) and torch.allclose(p, master[part], rtol=1e-4, atol=1e-6)
        at += g.numel()
