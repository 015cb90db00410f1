"""A bf16 gradient of the head is overwritten: a call that asks for it to be added to is refused."""
from __future__ import annotations

import pytest

from paper_2510_02483_amd import lib as L

UNSUPPORTED, WORKSPACE = 3, 6
A = 1 << 30  # addresses are compared, never followed, by a call that refuses


@pytest.mark.parametrize("dh", [None, 6 * A])
def test_accumulating_in_bf16_is_refused(dh):
    def bwd(accumulate, d_embed, low):
        return L.lib().ls_head_loss_bwd(100, 64, 1003, A, 2 * A, 3 * A, 4 * A, None, dh, d_embed, accumulate, low, 0, 8 * A, 0,
                                        None)

    assert bwd(1, None, 7 * A) == UNSUPPORTED and b"bf16" in L.lib().ls_last_error()
    # what is allowed gets as far as the workspace, which is too small
    assert bwd(0, None, 7 * A) == WORKSPACE and bwd(1, 7 * A, None) == WORKSPACE
