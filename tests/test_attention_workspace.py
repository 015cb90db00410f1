"""Where the attention backward's partial sums lie in its workspace."""
from __future__ import annotations

import ctypes

import pytest

from paper_2510_02483_amd import lib as L
from paper_2510_02483_amd.configs import B3


@pytest.mark.parametrize("nq,nkv", [(7, 1), (3, 1), (5, 5), (4, 2)])
@pytest.mark.parametrize("rows", [1, 3, 77, 1021, 4096])
@pytest.mark.parametrize("d", [64, 72, 128])
def test_partial_sums_start_at_a_multiple_of_256(rows, nq, nkv, d):
    """Behind D and the log-sum-exp, 8 bytes for each row and query head, an odd number of them here and there.  The sums
    are whole rows of [dK | dV] in fp32, 512 bytes at least, so the workspace's size tells where they start."""
    c = L.LsPackedCfg(rows, 3, nq, nkv, d)
    n = L.lib().ls_packed_attn_bwd_workspace(ctypes.byref(c))
    assert n >= 8 * rows * nq and n % 256 == 0
    if d != 72:
        n = L.ls_attn_core_bwd_workspace(B3.with_(batch=1, seq=rows, n_q_heads=nq, n_kv_heads=nkv, head_dim=d))
        assert n >= 8 * rows * nq and n % 256 == 0
