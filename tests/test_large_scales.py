"""Scales whose product with log2(e) is past fp32's range are refused: 0 times it would be no number."""
from __future__ import annotations

import ctypes
import math

import pytest
import torch

from gpu_util import need_gpu
from paper_2510_02483_amd import lib as L
from paper_2510_02483_amd.configs import ScoreConfig
from test_gpu_logprob import Head
from test_gpu_packed import Batch
from test_logprob import SHAPE, bwd, fwd
from test_post_training_checks import score_bwd, score_fwd

LARGE = [1.8e38, 2.4e38, 3.4e38]


@pytest.mark.parametrize("scale", LARGE)
def test_log_probabilities(scale):
    assert fwd(scale=scale) == SHAPE and bwd(scale=scale) == SHAPE


@pytest.mark.parametrize("scale", LARGE)
@pytest.mark.parametrize("window", [0, 5])
def test_scores(scale, window):
    sc = ctypes.byref(L.make_score_cfg(ScoreConfig(scale=scale, window=window)))
    assert score_fwd(sc) == SHAPE and score_bwd(sc) == SHAPE


@pytest.mark.gpu
def test_logits_of_zero_at_the_largest_scale():
    need_gpu()
    x = Head(20, 64, 300, 3, scale=2.0 ** 127, masked=0.0)
    x.h.zero_()
    x.dlp /= 2.0 ** 127
    x.den /= 2.0 ** 127
    x.fwd().bwd(x.de)
    assert float((x.logprob + math.log(300)).abs().max()) <= 2.0 ** -16
    assert (x.ids == torch.arange(3, device="cuda")).all()
    assert torch.isfinite(x.dh).all() and not x.de.any()


@pytest.mark.gpu
@pytest.mark.parametrize("window", [0, 5])
def test_scores_of_zero_at_the_largest_scale(window):
    need_gpu()
    b = Batch([200, 3], 2, 1, 64, seed=3)
    b.qkv[:, :128] = 0.0
    score = ScoreConfig(scale=2.0 ** 127, window=window)
    L.ls_packed_plan(b.c, b.cu, b.plan)
    L.ls_packed_score_attn_fwd(b.c, score, b.plan, b.qkv, b.o, b.lse)
    n = torch.arange(1, 201, device="cuda").clamp(max=window or 200)
    assert float((b.lse[0, :200] - torch.log(n.float())).abs().max()) <= 2.0 ** -16
