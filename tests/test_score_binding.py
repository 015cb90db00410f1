"""A window past 32 bits sees every position that one of 2^31 - 1 sees; cut to its low bits it would be another one."""
from __future__ import annotations

import pytest

from paper_2510_02483_amd import lib as L
from paper_2510_02483_amd.configs import ScoreConfig


@pytest.mark.parametrize("window,want", [(0, 0), (5, 5), (2 ** 31 - 1, 2 ** 31 - 1), (2 ** 31, 2 ** 31 - 1),
                                         (2 ** 32, 2 ** 31 - 1), (2 ** 32 + 5, 2 ** 31 - 1), (2 ** 63, 2 ** 31 - 1)])
def test_window(window, want):
    assert L.make_score_cfg(ScoreConfig(window=window)).window == want


@pytest.mark.parametrize("window", [-1, -2 ** 31, -2 ** 32 + 5, -2 ** 40])
def test_negative_windows_stay_negative(window):
    assert L.make_score_cfg(ScoreConfig(window=window)).window < 0
