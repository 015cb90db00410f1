"""Operators of post-training on buffers whose offsets pass 31 and 32 bits."""
from __future__ import annotations

import pytest
import torch

from gpu_util import bf16_randn
from paper_2510_02483_amd import lib as L
from paper_2510_02483_amd.configs import PackedConfig, ScoreConfig
from test_gpu_limits import need_memory
from test_gpu_logprob import I32, Head, check_top, within
from test_gpu_packed import Batch
from test_gpu_packed_score import check, run

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("cap", [0.0, 20.0])
def test_windowed_attention(cap):
    """qkv of 4.4 GB, o of 2.9: a short sequence behind a long one gives what it gives alone."""
    need_memory(40 << 30)
    nq, nkv, d, rows, live = 64, 16, 128, 180_000, 200
    score = ScoreConfig(cap=cap, window=100)
    small = run(Batch([live], nq, nkv, d, seed=3, std=1.5), score, rest=True)
    c = PackedConfig(rows, 2, nq, nkv, d)
    qkv = torch.zeros(rows, (nq + 2 * nkv) * d, dtype=torch.bfloat16, device="cuda")
    o, rest, dout = (torch.zeros(rows, nq * d, dtype=torch.bfloat16, device="cuda") for _ in range(3))
    assert qkv.numel() * 2 > 1 << 32 and o.numel() * 2 > 1 << 31
    qkv[-live:], dout[-live:] = small.qkv, small.dout
    lse, dqkv = torch.zeros(nq, rows, device="cuda"), torch.zeros_like(qkv)
    plan = torch.empty(L.ls_packed_plan_bytes(c), dtype=torch.uint8, device="cuda")
    ws = torch.empty(L.ls_packed_attn_bwd_workspace(c), dtype=torch.uint8, device="cuda")
    L.ls_packed_plan(c, torch.tensor([0, rows - live, rows], dtype=I32, device="cuda"), plan)
    L.ls_packed_score_attn_fwd(c, score, plan, qkv, o, lse, o_rest=rest)
    L.ls_packed_score_attn_bwd(c, score, plan, qkv, o, lse, dout, dqkv, ws, o_rest=rest)
    for a, b in ((o, small.o), (rest, small.rest), (dqkv[:, :nq * d], small.dqkv[:, :nq * d])):
        assert torch.equal(a[-live:], b)
    assert torch.equal(lse[:, -live:], small.lse)
    assert not o[:-live].any() and not dqkv[:-live].any()  # (values and gradients of 0)
    small.dqkv = dqkv[-live:]  # (dk and dv may be added in another order)
    check(small, score)


def test_alternatives():
    """2.3e9 maxima of groups, beside statistics of 2.3 GB: the last rows, and the last tokens of the vocabulary."""
    need_memory(30 << 30)
    T, H, V, top, few = 70_000, 8, 262_145, 5, 60
    groups = (V + 255) // 256 * 32
    assert T * groups > 1 << 31
    x = Head(T, H, V, top, seed=7, masked=0.0, std=1.0)
    x.t[-1] = V - 1
    ws = torch.empty(L.ls_token_logprob_workspace(T, H, V, top, 1), dtype=torch.uint8, device="cuda")
    assert ws.numel() > 4 * T * groups
    x.fwd(ws)
    y = Head(few, H, 64, top, masked=0.0)
    y.V, y.e = V, x.e
    for part in (slice(0, few), slice(T - few, T)):
        y.h, y.t, y.dlp, y.den = (a[part].contiguous() for a in (x.h, x.t, x.dlp, x.den))
        y.logprob, y.entropy, y.lse, y.ids, y.vals = (a[part] for a in (x.logprob, x.entropy, x.lse, x.ids, x.vals))
        r = y.reference()
        for name in ("lse", "logprob", "entropy"):
            within(name, getattr(y, name), r[name], r["tol_" + name] + 2.0 ** -14)  # (logits up to 60)
        check_top(y, r)


def test_gradients_of_more_than_2_31_elements():
    need_memory(20 << 30)
    n = (1 << 31) + 20_003
    g = torch.zeros(n, dtype=torch.bfloat16, device="cuda")
    small = torch.ones(5, device="cuda")
    for at, v in ((0, 3.0), (1 << 30, 1.0), ((1 << 31) - 1, 2.0), (1 << 31, 4.0), (n - 1, 5.0)):
        g[at] = v
    norm, ws = torch.zeros(1, device="cuda"), torch.empty(L.ls_grad_norm_workspace(), dtype=torch.uint8, device="cuda")
    L.ls_grad_norm([small, g], norm, ws)
    want = 60.0 ** 0.5  # 9 + 1 + 4 + 16 + 25 + 5
    assert abs(norm.item() - want) <= 2.0 ** -23 * want
    L.ls_grad_clip([small, g], norm, want / 2)
    for at, v in ((0, 1.5), (1 << 30, 0.5), ((1 << 31) - 1, 1.0), (1 << 31, 2.0), (n - 1, 2.5)):
        assert abs(g[at].item() - v) <= 2.0 ** -8 * v
    assert int((g[(1 << 31) - 100:] != 0).sum()) == 3
    out = [torch.full_like(small, 9.0), torch.full_like(g, 9.0)]
    L.ls_grad_clip([small, g], norm, 100.0, out)
    assert torch.equal(out[0], small) and torch.equal(out[1], g)
