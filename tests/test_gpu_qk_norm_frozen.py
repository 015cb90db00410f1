"""The backward pass of the q/k norm with both gains frozen, which needs no workspace."""
from __future__ import annotations

import pytest
import torch

from gpu_util import need_gpu
from paper_2510_02483_amd import lib as L
from test_gpu_packed import Batch
from test_gpu_qk_norm import Norm

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("nbytes", [None, 16])
def test_no_workspace(nbytes):
    need_gpu()
    n = Norm(Batch([50, 0, 1, 333], 4, 2, 64, tail=3, seed=11)).bwd()
    dx = n.dx.clone()
    n.dx.fill_(77.0)
    n.ws = None if nbytes is None else torch.full((nbytes,), 9, dtype=torch.uint8, device="cuda")
    n.bwd(dgq=None, dgk=None)
    assert torch.equal(n.dx, dx)
    assert nbytes is None or (n.ws == 9).all()
    for gains in (dict(dgq=None), dict(dgk=None)):
        with pytest.raises(L.LsError):
            n.bwd(**gains)
