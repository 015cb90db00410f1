"""README's example of a policy-gradient step on packed documents, as it stands there, on buffers that served another batch."""
from __future__ import annotations

import re

import numpy as np
import pytest
import torch

import packed_ref as R
from gpu_util import bf16_randn, f64, need_gpu
from paper_2510_02483_amd import lib
from paper_2510_02483_amd.configs import PackedConfig, ScoreConfig
from test_gpu_readme import NKV, NQ, D, H, README, V

pytestmark = pytest.mark.gpu


def example():
    return next(b for b in re.findall(r"```python\n(.*?)```", open(README).read(), re.S) if "ls_token_logprob_fwd" in b)


def buffers(T, fill):
    def new(*s, dt=torch.bfloat16):
        return torch.full(s, fill, dtype=dt, device="cuda")

    f, n = torch.float32, (NQ + 2 * NKV) * D
    return dict(y=new(T, n), dy=new(T, n), dqkv=new(T, n), o=new(T, NQ * D), o_rest=new(T, NQ * D), lse=new(NQ, T, dt=f),
                logprob=new(T, dt=f), entropy=new(T, dt=f), head_lse=new(T, dt=f), dh=new(T, H), d_embed=new(V, H, dt=f),
                dq_gain=new(D, dt=f), dk_gain=new(D, dt=f), norm=new(1, dt=f))


def step(T, docs, out, seed):
    """The example, and the two weight gradients behind it that sum over all rows."""
    cu = R.bounds_of(docs)
    live = int(cu[-1])
    rng = np.random.default_rng(seed)
    targets = torch.full((T,), -1, dtype=torch.int32)
    targets[:live] = torch.from_numpy(rng.integers(-1, V, live).astype(np.int32))

    def rows(scale):
        return torch.from_numpy((rng.standard_normal(T) * scale).astype(np.float32)).cuda()

    def space(n):
        return torch.empty(n, dtype=torch.uint8, device="cuda")

    c = PackedConfig(T, len(docs), NQ, NKV, D)
    s = dict(out, lib=lib, ScoreConfig=ScoreConfig, c=c, live=live, temperature=0.8, targets=targets.cuda(),
             plan=space(lib.ls_packed_plan_bytes(c)), qkv=bf16_randn((T, (NQ + 2 * NKV) * D), seed),
             do=bf16_randn((T, NQ * D), seed + 1), h=bf16_randn((T, H), seed + 2), embed=bf16_randn((V, H), seed + 3, 0.05),
             q_gain=bf16_randn((D,), seed + 4) + 1, k_gain=bf16_randn((D,), seed + 5) + 1, dlogprob=rows(0.1),
             dentropy=rows(0.01), grads=[out["d_embed"], out["dq_gain"], out["dk_gain"]],
             workspace=space(lib.ls_token_logprob_workspace(T, H, V)), attn_workspace=space(lib.ls_packed_attn_bwd_workspace(c)),
             qk_workspace=space(lib.ls_packed_qk_norm_rope_bwd_workspace(c)), norm_workspace=space(lib.ls_grad_norm_workspace()))
    lib.ls_packed_plan(c, torch.tensor(cu, dtype=torch.int32, device="cuda"), s["plan"])
    exec(example(), s)
    grads = {"wqkv": torch.empty((NQ + 2 * NKV) * D, H, device="cuda"), "wo": torch.empty(H, NQ * D, device="cuda")}
    lib.ls_gemm_tn(s["dqkv"], s["h"], grads["wqkv"])
    lib.ls_gemm_tn(s["dh"], s["o"], grads["wo"])
    grads.update({k: s[k] for k in ("d_embed", "dq_gain", "dk_gain", "norm")})
    return s, grads


def test_example_on_buffers_of_an_earlier_batch():
    need_gpu()
    T = 256
    out = buffers(T, float("nan"))
    step(T, [100, 156], out, 61)
    for k in ("y", "dy", "o", "o_rest", "dqkv"):  # (whatever an earlier batch left there)
        out[k][160:] = float("nan")
    s, grads = step(T, [70, 0, 90], out, 71)
    assert s["dqkv"] is out["dqkv"]
    fresh, want = step(T, [70, 0, 90], buffers(T, 0.0), 71)
    for k in grads:
        assert torch.isfinite(grads[k]).all() and torch.equal(grads[k], want[k]), k
    live = s["live"]
    for k in ("o", "dqkv", "dh", "logprob", "entropy"):
        assert not s[k][live:].any() and torch.equal(s[k], fresh[k]), k
    x, y = f64(s["dqkv"])[:live], f64(s["h"])[:live]
    assert np.all(np.abs(f64(grads["wqkv"]) - x.T @ y) <= 2 * T * R.W * (np.abs(x).T @ np.abs(y)))
