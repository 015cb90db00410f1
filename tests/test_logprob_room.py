"""What the forward call of the log probabilities needs of its workspace, where the backward call's share is small."""
from __future__ import annotations

import pytest

from test_logprob import WORKSPACE, fwd, need


@pytest.mark.parametrize("T,H,V", [(1, 8, 20003), (15, 8, 20003), (17, 8, 20003), (1027, 8, 20003), (4096, 64, 100_000)])
def test_the_alternatives_room(T, H, V):
    """4 bytes for every 8 logits, in rows of 16 (or as many as there are) and whole tiles of 256 columns; as much for
    any number of alternatives.  The forward call needs all of it."""
    plain = need(T, H, V, 0, 1)
    for top in (1, 5, 64):
        n = need(T, H, V, top, 1)
        rows = next(r for r in (1, 2, 4, 8, 16) if r >= min(T, 16))
        room = -(-T // rows) * rows * (-(-V // 256) * 32) * 4
        assert room >= -(-V // 8) * T * 4
        assert plain < n and room < n <= room + plain + 512
        assert fwd(T, H, V, top=top, n=n - 256) == WORKSPACE
