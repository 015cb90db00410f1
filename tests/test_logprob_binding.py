"""Buffers of alternatives whose rows are not the tokens': another number of columns would be read from them than they have."""
from __future__ import annotations

import pytest
import torch

from paper_2510_02483_amd import lib as L

T, H, V = 4, 8, 30
F32, I32, BF16 = torch.float32, torch.int32, torch.bfloat16


def call(ids, vals):
    row = torch.zeros(T)
    L.ls_token_logprob_fwd(torch.zeros(T, H, dtype=BF16), torch.zeros(V, H, dtype=BF16), torch.zeros(T, dtype=I32), row, row,
                           row, torch.zeros(64, dtype=torch.uint8), top_ids=torch.zeros(ids, dtype=I32),
                           top_logprob=torch.zeros(vals))


@pytest.mark.parametrize("ids,vals", [((8, 5), (8, 5)), ((2, 10), (2, 10)), ((4, 5), (5, 4)), ((5, 4), (4, 5)), ((2, 4, 5), (2, 4, 5)),
                                      ((20,), (2, 10)), ((4, 0), (4, 0)), ((4, 5), (4, 4))])
def test_another_shape_is_refused(ids, vals):
    with pytest.raises(ValueError, match="top_ids and top_logprob"):
        call(ids, vals)


@pytest.mark.parametrize("shape", [(4, 5), (4, 1), (2, 2, 5), (20,)])
def test_the_tokens_rows_are_taken(shape):
    with pytest.raises(ValueError, match="GPU"):  # (as far as the check of the device)
        call(shape, shape)
