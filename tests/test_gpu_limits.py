"""Sizes at the far end of what the packed operators accept."""
from __future__ import annotations

import pytest
import torch

import packed_ref as R
from gpu_util import need_gpu
from paper_2510_02483_amd import lib as L
from paper_2510_02483_amd.configs import PackedConfig
from test_gpu_packed import MARK, Batch, check

pytestmark = pytest.mark.gpu


def need_memory(nbytes):
    need_gpu()
    torch.cuda.empty_cache()
    if torch.cuda.mem_get_info()[0] < nbytes:
        pytest.skip(f"needs {nbytes >> 30} GiB of free device memory")


def test_packed_rows_beyond_one_dimension_of_a_launch():
    """2^26 rows with room for as many sequences: 18.1 million workgroups of 256 threads in the forward and in the dK/dV
    kernel, 2^24 where D is formed; one dimension of a launch holds fewer than 2^24.  The sequences lie at the far
    end, whose D the last workgroups form."""
    need_memory(100 << 30)
    lens, d = [150, 65, 0, 33, 7, 64], 64
    total = n_seqs = 1 << 26
    small = Batch(lens, 1, 1, d, seed=41).run()
    rows = sum(lens)
    first = total - rows
    c = PackedConfig(total, n_seqs, 1, 1, d)
    cu = torch.full((n_seqs + 1,), first, dtype=torch.int32, device="cuda")
    cu[-len(lens) - 1:] = torch.tensor(R.bounds_of(lens, first), dtype=torch.int32)
    plan = torch.empty(L.ls_packed_plan_bytes(c), dtype=torch.uint8, device="cuda")
    qkv, dout = (torch.zeros(total, k * d, dtype=torch.bfloat16, device="cuda") for k in (3, 1))
    qkv[first:], dout[first:] = small.qkv, small.dout
    o, dqkv = torch.full_like(dout, MARK), torch.full_like(qkv, MARK)
    lse = torch.full((1, total), MARK, device="cuda")
    L.ls_packed_plan(c, cu, plan)
    L.ls_packed_attn_fwd(c, plan, qkv, o, lse)
    ws = torch.empty(L.ls_packed_attn_bwd_workspace(c), dtype=torch.uint8, device="cuda")
    L.ls_packed_attn_bwd(c, plan, qkv, o, lse, dout, dqkv, ws)
    assert torch.equal(o[first:], small.o) and torch.equal(lse[:, first:], small.lse)
    assert torch.equal(dqkv[first:, :d], small.dqkv[:, :d])
    small.dqkv = dqkv[first:]  # dk and dv of a long row's plan may be added in another order
    check(small)
    assert bool((lse[:, :first] == MARK).all())
    for t in (o, dqkv):
        for a in range(0, first, 1 << 23):
            assert bool((t[a:min(a + (1 << 23), first)] == MARK).all())

@pytest.mark.parametrize("heads", [256, 300, 512, 513, 700])
def test_more_kv_heads_than_parts(heads):
    """Beyond 512 kv heads no tile is cut and no partial sums are joined."""
    need_gpu()
    check(Batch([60, 1, 0, 30], heads, heads, 64, first=1, tail=2, seed=43).run())
