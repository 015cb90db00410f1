"""The room that the alternatives of the log probabilities take in a workspace, between guards."""
from __future__ import annotations

import pytest
import torch

from gpu_util import need_gpu
from paper_2510_02483_amd import lib as L
from test_gpu_logprob import F32, I32, Head, check_fwd, full

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("T", [1, 15, 16, 17, 130, 600, 1027])
@pytest.mark.parametrize("H,V,top", [(8, 20003, 5), (16, 4099, 64), (8, 257, 1), (8, 1, 3)])
def test_room_of_the_alternatives(T, H, V, top):
    """A forward call in as many bytes as small pieces of the backward call leave to it, between guards."""
    need_gpu()
    x = Head(T, H, V, top, seed=T + V, masked=0.0)
    n = L.ls_token_logprob_workspace(T, H, V, top, 1)
    pad = 1 << 16
    room = torch.full((n + 2 * pad,), 9, dtype=torch.uint8, device="cuda")
    outs = {}
    for name, k, dt in (("ids", T * top, I32), ("vals", T * top, F32), ("logprob", T, F32), ("entropy", T, F32), ("lse", T, F32)):
        outs[name] = full(k + 4096, dtype=dt)
        setattr(x, name, outs[name][:k].view(getattr(x, name).shape))
    for fill in (9, 255, 0):
        room[pad:pad + n] = fill
        x.fwd(room[pad:pad + n])
        assert (room[:pad] == 9).all() and (room[pad + n:] == 9).all()
    for name, t in outs.items():
        assert (t[-4096:] == 7).all(), name
    check_fwd(x, x.reference())
