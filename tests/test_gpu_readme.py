"""README's example of training on packed documents, as it stands there, on buffers that served another batch."""
from __future__ import annotations

import os
import re

import numpy as np
import pytest
import torch

import packed_ref as R
from gpu_util import bf16_randn, f64, need_gpu
from paper_2510_02483_amd import lib
from paper_2510_02483_amd.configs import PackedConfig

pytestmark = pytest.mark.gpu

README = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "README.md")
NQ, NKV, D, H, V = 24, 8, 128, 256, 1000  # the heads of the example


def example():
    return next(b for b in re.findall(r"```python\n(.*?)```", open(README).read(), re.S) if "ls_packed_plan" in b)


def buffers(T, fill):
    def new(*s, dt=torch.bfloat16):
        return torch.full(s, fill, dtype=dt, device="cuda")

    f = torch.float32
    return dict(o=new(T, NQ * D), lse=new(NQ, T, dt=f), dqkv=new(T, (NQ + 2 * NKV) * D), loss=new(1, dt=f),
                row_loss=new(T, dt=f), head_lse=new(T, dt=f), dh=new(T, H), d_embed=new(V, H, dt=f))


def step(T, docs, out, seed):
    """The example, and the two weight gradients behind it that sum over all rows."""
    cu = R.bounds_of(docs)
    live = int(cu[-1])
    targets = torch.full((T,), -1, dtype=torch.int32)
    targets[:live] = torch.from_numpy(np.random.default_rng(seed).integers(0, V, live).astype(np.int32))
    s = dict(out, torch=torch, lib=lib, PackedConfig=PackedConfig, T=T, docs=docs, live=live,
             cu_seqlens=torch.tensor(cu, dtype=torch.int32, device="cuda"), targets=targets.cuda(),
             qkv=bf16_randn((T, (NQ + 2 * NKV) * D), seed), do=bf16_randn((T, NQ * D), seed + 1),
             h=bf16_randn((T, H), seed + 2), embed=bf16_randn((V, H), seed + 3, 0.05),
             workspace=torch.empty(lib.ls_head_loss_workspace(T, H, V), dtype=torch.uint8, device="cuda"))
    c = PackedConfig(T, len(docs), NQ, NKV, D)
    s["attn_workspace"] = torch.empty(lib.ls_packed_attn_bwd_workspace(c), dtype=torch.uint8, device="cuda")
    exec(example(), s)
    grads = {"wqkv": torch.empty((NQ + 2 * NKV) * D, H, device="cuda"), "wo": torch.empty(H, NQ * D, device="cuda")}
    lib.ls_gemm_tn(s["dqkv"], s["h"], grads["wqkv"])
    lib.ls_gemm_tn(s["dh"], s["o"], grads["wo"])
    return s, grads


def test_example_on_buffers_of_an_earlier_batch():
    need_gpu()
    T = 256
    out = buffers(T, float("nan"))
    step(T, [100, 156], out, 61)
    s, grads = step(T, [70, 0, 90], out, 71)
    assert s["dqkv"] is out["dqkv"]
    fresh, want = step(T, [70, 0, 90], buffers(T, 0.0), 71)
    for k in grads:
        assert torch.equal(grads[k], want[k]), k
    live = s["live"]
    for k in ("o", "dqkv", "dh"):
        assert not s[k][live:].any() and torch.equal(s[k], fresh[k])
    # and the gradient is that of the documents alone; fp32 sums of 256 terms
    x, y = f64(s["dqkv"])[:live], f64(s["h"])[:live]
    assert np.all(np.abs(f64(grads["wqkv"]) - x.T @ y) <= 2 * T * R.W * (np.abs(x).T @ np.abs(y)))
