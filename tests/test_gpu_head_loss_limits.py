"""The head loss where the tiles of one product over the vocabulary would be more than a launch's dimension holds."""
from __future__ import annotations

import torch

import pytest
from paper_2510_02483_amd import lib as L
from test_gpu_head_loss import W, within
from test_gpu_limits import need_memory

pytestmark = pytest.mark.gpu


def test_more_tiles_than_one_dimension_of_a_launch():
    """2^23 tokens and 131072 entries: 2^24 tiles of 256 x 256, each 256 threads."""
    need_memory(90 << 30)
    T, H, V = 1 << 23, 8, 131072
    g = torch.Generator(device="cuda")
    g.manual_seed(45)
    h = torch.randn(T, H, generator=g, device="cuda").bfloat16()
    e = torch.randn(V, H, generator=g, device="cuda").bfloat16()
    t = torch.randint(0, V, (T,), generator=g, device="cuda", dtype=torch.int32)
    loss, rows, lse = (torch.full((n,), float("nan"), device="cuda") for n in (1, T, T))
    ws = torch.empty(L.ls_head_loss_workspace(T, H, V), dtype=torch.uint8, device="cuda")
    L.ls_head_loss_fwd(h, e, t, loss, rows, lse, ws)
    at = torch.cat([torch.arange(a, a + 32, device="cuda") for a in (0, T // 2 - 16, T - 32)])
    x, e64 = h[at].double(), e.double()
    z = x @ e64.T
    ref = torch.logsumexp(z, 1)
    ez = H * W * (x.abs() @ e64.abs().T).amax(1)
    tol = ez + 2.0 ** -17 + 2.0 ** -21 * ref.abs()  # as in test_gpu_head_loss
    within("lse", lse[at], ref, tol)
    within("row_loss", rows[at], ref - z.gather(1, t[at].long()[:, None])[:, 0], tol + ez)
    assert bool(torch.isfinite(rows).all())
    # a sum of row losses in fp64, rounded once to fp32
    mean = float(rows.double().mean())
    assert abs(loss.item() - mean) <= 2.0 ** -23 * abs(mean)
