"""What the lengths of the other sequences of a row may change in a sequence's results, and what not."""
from __future__ import annotations

import pytest
import torch

from gpu_util import need_gpu
from test_gpu_packed import Batch, check

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("nq,nkv,d", [(8, 2, 64), (8, 1, 128), (4, 1, 104), (2, 2, 64)])
@pytest.mark.parametrize("rows", [1, 17, 32, 33, 64])
def test_short_among_few_and_among_many(rows, nq, nkv, d):
    """Few sequences of up to 64 rows are listed as tiles where a kv head has more than two query heads, many are not: o,
    lse and dq are the same bits, dk and dv within their bounds."""
    need_gpu()
    few = Batch([rows, 200], nq, nkv, d, seed=51)
    many = Batch([rows] + [5] * (64 // nkv + 1) + [200], nq, nkv, d, seed=51)
    many.qkv[:rows], many.dout[:rows] = few.qkv[:rows], few.dout[:rows]
    few.run()
    many.run()
    assert torch.equal(few.o[:rows], many.o[:rows]) and torch.equal(few.lse[:, :rows], many.lse[:, :rows])
    assert torch.equal(few.dqkv[:rows, :nq * d], many.dqkv[:rows, :nq * d])
    check(few)
    check(many)


@pytest.mark.parametrize("nq,nkv,d", [(8, 1, 64), (4, 2, 128)])
def test_tiles_among_short_and_among_long(nq, nkv, d):
    """The same of a sequence of several tiles, alone and beside one that makes its share of the work small."""
    need_gpu()
    rows = 300
    alone = Batch([rows], nq, nkv, d, seed=53)
    beside = Batch([rows, 2000, 3], nq, nkv, d, seed=53)
    beside.qkv[:rows], beside.dout[:rows] = alone.qkv[:rows], alone.dout[:rows]
    alone.run()
    beside.run()
    assert torch.equal(alone.o[:rows], beside.o[:rows]) and torch.equal(alone.lse[:, :rows], beside.lse[:, :rows])
    assert torch.equal(alone.dqkv[:rows, :nq * d], beside.dqkv[:rows, :nq * d])
    check(alone)
    check(beside)
