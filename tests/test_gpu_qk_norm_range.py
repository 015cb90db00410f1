"""q/k norm of heads whose squares leave the range of 32 bits, against the 64-bit reference of score_ref."""
from __future__ import annotations

import numpy as np
import pytest
import torch

from gpu_util import f64, need_gpu, say
from test_gpu_packed import Batch
from test_gpu_qk_norm import Norm

pytestmark = pytest.mark.gpu
STEP = 1.01 * 2.0 ** -134  # half a step between the type's smallest values


def times(t, m):
    """t m, rounded on the host: smallest values are kept."""
    return (t.cpu().double() * m).to(torch.bfloat16).cuda()


def check(n):
    v = (n.b.nq + n.b.nkv) * n.b.d
    for name, got, (ref, lim) in zip(("y", "dx", "dgq", "dgk"), (n.y, n.dx, n.dgq, n.dgk), n.want()):
        got = f64(got)
        if got.ndim == 2:
            got, ref, lim = got[:, :v], ref[:, :v], lim[:, :v] + STEP
        assert np.abs(ref).max() < 3e38
        err = np.abs(got - ref)
        assert np.all(err <= lim), (name, float(np.nanmax(err / lim)), int((~(err <= lim)).sum()))
        say(f"{name}: worst share of the bound {np.max(err / lim):.2f}")


# the size of x, eps, the size of dy (so that dx, of the size of dy / x, can be held)
SIZES = [(2.0 ** 124, 1e-5, 1.0), (2.0 ** 124, 0.0, 2.0 ** 100), (2.0 ** 66, 1e-5, 1.0), (2.0 ** 62, 1e-5, 1.0),
         (2.0 ** -45, 0.0, 1.0), (2.0 ** -50, 1e-30, 1.0), (2.0 ** -60, 0.0, 1.0), (2.0 ** -70, 0.0, 1.0),
         (2.0 ** -80, 1e-38, 2.0 ** -20), (2.0 ** -120, 0.0, 2.0 ** -60), (2.0 ** -120, 1e-36, 2.0 ** -60),
         (2.0 ** -130, 0.0, 2.0 ** -60), (2.0 ** -126, 1e-30, 2.0 ** -60), (3e36, 3e38, 1.0)]


@pytest.mark.parametrize("nq,nkv,d", [(3, 1, 64), (8, 2, 128), (5, 1, 72), (2, 1, 80)])
@pytest.mark.parametrize("size,eps,dy", SIZES)
def test_heads_of_any_size(size, eps, dy, nq, nkv, d):
    need_gpu()
    n = Norm(Batch([40, 9], nq, nkv, d, seed=13), eps=eps)
    n.b.qkv = times(n.b.qkv, size)
    n.dy = times(n.dy, dy)
    n.fwd().bwd()
    check(n)


@pytest.mark.parametrize("nq,nkv,d", [(8, 8, 64), (8, 8, 128), (16, 2, 72)])
def test_a_head_s_size_is_its_own(nq, nkv, d):
    """Heads of ordinary sizes next to others that are not: their results are the same to the bit."""
    need_gpu()
    a, b = (Norm(Batch([40, 9], nq, nkv, d, seed=13), eps=1e-6) for _ in range(2))
    far = torch.zeros(nq + 2 * nkv, dtype=torch.bool)
    far[[0, 3, nq - 1, nq]] = True
    heads = b.b.qkv.view(49, -1, d)
    heads[::2, far] = times(heads[::2, far], 2.0 ** 110)
    heads[1::4, far] = times(heads[1::4, far], 2.0 ** -90)
    a.fwd().bwd(), b.fwd().bwd()
    for x, y in ((a.y, b.y), (a.dx, b.dx)):
        x, y = x.view(49, -1, d), y.view(49, -1, d)
        assert torch.equal(x[:, ~far], y[:, ~far]) and torch.equal(x[3::4], y[3::4])
    check(b)


def test_heads_without_a_size():
    """0 / 0 where eps is 0 too; infinities and NaN stay in their head."""
    need_gpu()
    n = Norm(Batch([40], 4, 1, 64, seed=13), eps=0.0)
    x = n.b.qkv.view(40, 6, 64)
    x[5, 1] = 0.0
    x[6, 2, 7] = float("inf")
    x[7, 4, 9] = float("nan")
    n.fwd().bwd(dgq=None, dgk=None)
    bad = torch.zeros(40, 6, dtype=torch.bool, device="cuda")
    bad[5, 1] = bad[6, 2] = bad[7, 4] = True
    for t in (n.y, n.dx):
        t = t.view(40, 6, 64)
        assert torch.equal(torch.isnan(t).any(2), bad)
        assert torch.isfinite(t[~bad]).all()
    assert torch.isnan(n.y.view(40, 6, 64)[5, 1]).all() and torch.isnan(n.y.view(40, 6, 64)[7, 4]).all()


@pytest.mark.parametrize("d", [64, 128])
def test_in_place(d):
    need_gpu()
    n = Norm(Batch([40, 9], 4, 2, d, seed=13), eps=1e-5)
    n.b.qkv = times(n.b.qkv, 2.0 ** 90)
    n.fwd().bwd()
    work, dwork = n.b.qkv.clone(), n.dy.clone()
    n.fwd(work, work).bwd(dwork, dwork)
    assert torch.equal(work, n.y) and torch.equal(dwork, n.dx)
