"""A training step on packed documents with the operators together, as a program uses them: embedding, RMSNorm,
projection, rotation, attention, output projection with the residual, RMSNorm and the tied head's loss, and all the
way back, against the same model in 64 bits by automatic differentiation."""
from __future__ import annotations

import numpy as np
import pytest
import torch

import packed_ref as R
from gpu_util import GRAD_TOL, OUT_TOL, bf16_randn, need_gpu, say
from paper_2510_02483_amd import lib as L
from paper_2510_02483_amd.configs import PackedConfig

pytestmark = pytest.mark.gpu

H, NQ, NKV, D, V, THETA, EPS = 256, 4, 2, 64, 1003, 1e4, 1e-5
LENS, TAIL = [70, 1, 0, 130, 33, 9, 50], 11


def model64(ids, targets, w, cu):
    """Loss of the one-layer model in float64, document by document."""
    x = w["embed"][ids]

    def norm(y, g):
        return y * (y.pow(2).mean(-1, keepdim=True) + EPS).rsqrt() * g

    qkv = norm(x, w["g1"]) @ w["wqkv"].T
    freq = THETA ** (-2.0 * torch.arange(D // 2, dtype=torch.float64, device=x.device) / D)
    outs = []
    for a, b in zip(cu, cu[1:]):
        n = b - a
        if n == 0:
            continue
        ang = torch.outer(torch.arange(n, dtype=torch.float64, device=x.device), freq)
        c, s = ang.cos(), ang.sin()
        y = qkv[a:b].view(n, NQ + 2 * NKV, D)

        def turn(z):
            lo, hi = z[..., :D // 2], z[..., D // 2:]
            return torch.cat([lo * c[:, None] - hi * s[:, None], lo * s[:, None] + hi * c[:, None]], -1)

        q, k, v = turn(y[:, :NQ]), turn(y[:, NQ:NQ + NKV]), y[:, NQ + NKV:]
        k, v = (z.repeat_interleave(NQ // NKV, 1) for z in (k, v))
        sc = torch.einsum("qhd,khd->hqk", q, k) / D ** 0.5
        sc = sc.masked_fill(torch.triu(torch.ones(n, n, dtype=torch.bool, device=x.device), 1), float("-inf"))
        outs.append(torch.einsum("hqk,khd->qhd", sc.softmax(-1), v).reshape(n, NQ * D))
    live = cu[-1]
    x2 = x[:live] + torch.cat(outs) @ w["wo"].T
    z = norm(x2, w["g2"]) @ w["embed"].T
    return torch.nn.functional.cross_entropy(z, targets[:live].long(), ignore_index=-1)


def test_step_on_packed_documents():
    need_gpu()
    cu = R.bounds_of(LENS)
    T = int(cu[-1]) + TAIL
    assert T % 8 == 0  # what the plain matrix products take
    g = torch.Generator().manual_seed(3)
    ids = torch.randint(0, V, (T,), generator=g, dtype=torch.int32)
    targets = torch.full((T,), -1, dtype=torch.int32)
    for a, b in zip(cu, cu[1:]):  # the next token of the same document
        if b - a > 1:
            targets[a:b - 1] = ids[a + 1:b]
    ids, targets = ids.cuda(), targets.cuda()
    w = dict(embed=bf16_randn((V, H), 1, 0.3), wqkv=bf16_randn(((NQ + 2 * NKV) * D, H), 2, 0.08),
             wo=bf16_randn((H, NQ * D), 3, 0.08), g1=bf16_randn((H,), 4, 0.1) + 1, g2=bf16_randn((H,), 5, 0.1) + 1)

    def new(*s, dt=torch.bfloat16):
        return torch.empty(*s, dtype=dt, device="cuda")

    f32 = torch.float32
    c = PackedConfig(T, len(LENS), NQ, NKV, D)
    plan = new(L.ls_packed_plan_bytes(c), dt=torch.uint8)
    L.ls_packed_plan(c, torch.tensor(cu, dtype=torch.int32, device="cuda"), plan)
    x, h1, r1 = new(T, H), new(T, H), new(T, dt=f32)
    L.ls_embed_fwd(ids, w["embed"], x)
    L.ls_rmsnorm_fwd(T, H, EPS, x, w["g1"], h1, r1)
    qkv = new(T, (NQ + 2 * NKV) * D)
    L.ls_gemm_nt(h1, w["wqkv"], qkv)
    L.ls_packed_rope(c, plan, THETA, qkv, qkv)
    o, lse = torch.full((T, NQ * D), float("nan"), dtype=torch.bfloat16, device="cuda"), new(NQ, T, dt=f32)
    L.ls_packed_attn_fwd(c, plan, qkv, o, lse)
    proj = new(T, H)
    L.ls_gemm_nt(o, w["wo"], proj)  # rows of no document hold NaN from here on
    x2 = x + proj
    h2, r2 = new(T, H), new(T, dt=f32)
    L.ls_rmsnorm_fwd(T, H, EPS, x2, w["g2"], h2, r2)
    loss, rows, lse2 = new(1, dt=f32), new(T, dt=f32), new(T, dt=f32)
    ws = new(L.ls_head_loss_workspace(T, H, V), dt=torch.uint8)
    L.ls_head_loss_fwd(h2, w["embed"], targets, loss, rows, lse2, ws)

    d = dict(embed=new(V, H, dt=f32), wqkv=new((NQ + 2 * NKV) * D, H, dt=f32), wo=new(H, NQ * D, dt=f32),
             g1=new(H, dt=f32), g2=new(H, dt=f32))
    dh2, dx2, dx = new(T, H), new(T, H), new(T, H)
    L.ls_head_loss_bwd(h2, w["embed"], targets, lse2, None, dh2, d["embed"], False, ws)
    live = int(cu[-1])
    assert not dh2[live:].any()
    # a program's own rows: the padding's activations are no numbers, its gradients are zero
    for t in (x2, r2, h1, r1, o):
        t[live:] = 0
    nw = new(L.ls_rmsnorm_bwd_workspace(T, H), dt=torch.uint8)
    L.ls_rmsnorm_bwd(T, H, x2, w["g2"], r2, dh2, None, dx2, d["g2"], False, nw)
    do = new(T, NQ * D)
    L.ls_gemm_nn(dx2, w["wo"], do)
    L.ls_gemm_tn(dx2, o, d["wo"])
    dqkv = torch.zeros_like(qkv)
    L.ls_packed_attn_bwd(c, plan, qkv, o, lse, do, dqkv,
                         new(L.ls_packed_attn_bwd_workspace(c), dt=torch.uint8))
    L.ls_packed_rope(c, plan, THETA, dqkv, dqkv, inverse=True)
    dh1 = new(T, H)
    L.ls_gemm_nn(dqkv, w["wqkv"], dh1)
    L.ls_gemm_tn(dqkv, h1, d["wqkv"])
    L.ls_rmsnorm_bwd(T, H, x, w["g1"], r1, dh1, dx2, dx, d["g1"], False, nw)
    L.ls_embed_bwd(ids, dx, d["embed"])

    w64 = {k: t.double().requires_grad_() for k, t in w.items()}
    ref = model64(ids.long(), targets, w64, [int(v) for v in cu])
    ref.backward()
    say(f"loss {loss.item():.6f} against {ref.item():.6f}")
    assert abs(loss.item() - ref.item()) <= OUT_TOL * abs(ref.item())
    for k, t in w64.items():
        rel = float((d[k].double() - t.grad).norm() / t.grad.norm())
        say(f"{k}: {rel:.2e}")
        assert rel <= GRAD_TOL, k
    assert np.isfinite(float(sum(t.abs().sum() for t in d.values())))
