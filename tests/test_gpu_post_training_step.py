"""A policy-gradient step on packed samples with its operators together, as a program uses them: projection, q/k norm with
rotation, attention with capped scores and a window, output projection with the residual, RMSNorm, log probabilities and
entropies under the head, all the way back, and the gradients clipped by their common norm, against the same model
in 64 bits by automatic differentiation."""
from __future__ import annotations

import pytest
import torch

import packed_ref as R
from gpu_util import GRAD_TOL, OUT_TOL, bf16_randn, need_gpu, say
from paper_2510_02483_amd import lib as L
from paper_2510_02483_amd.configs import PackedConfig, ScoreConfig

pytestmark = pytest.mark.gpu

H, NQ, NKV, D, V, THETA, EPS, SCALE, CAP, WINDOW = 256, 4, 2, 64, 1003, 1e4, 1e-5, 1.25, 20.0, 40
LENS, TAIL = [70, 1, 0, 130, 33, 9, 50], 11
BF16, F32 = torch.bfloat16, torch.float32


def model64(x, targets, adv, ent, w, cu):
    """The objective in float64, document by document, and the log probabilities and entropies."""
    def norm(y, g):
        return y * (y.pow(2).mean(-1, keepdim=True) + EPS).rsqrt() * g

    qkv = x @ w["wqkv"].T
    freq = THETA ** (-2.0 * torch.arange(D // 2, dtype=torch.float64, device=x.device) / D)
    outs = []
    for a, b in zip(cu, cu[1:]):
        n = b - a
        if n == 0:
            continue
        ang = torch.outer(torch.arange(n, dtype=torch.float64, device=x.device), freq)
        c, s = ang.cos()[:, None], ang.sin()[:, None]
        y = qkv[a:b].view(n, NQ + 2 * NKV, D)

        def turn(z):
            lo, hi = z[..., :D // 2], z[..., D // 2:]
            return torch.cat([lo * c - hi * s, lo * s + hi * c], -1)

        q, k, v = turn(norm(y[:, :NQ], w["gq"])), turn(norm(y[:, NQ:NQ + NKV], w["gk"])), y[:, NQ + NKV:]
        i = torch.arange(n, device=x.device)
        far = i[:, None] - i[None, :]
        o = []
        for h in range(NQ):
            sc = CAP * torch.tanh(q[:, h] @ k[:, h // 2].T / D ** 0.5 / CAP)
            sc = sc.masked_fill((far < 0) | (far >= WINDOW), float("-inf"))
            o.append(sc.softmax(-1) @ v[:, h // 2])
        outs.append(torch.cat(o, 1))
    live = cu[-1]
    h2 = norm(x[:live] + torch.cat(outs) @ w["wo"].T, w["g2"])
    ln = torch.log_softmax(h2 @ w["embed"].T * SCALE, 1)
    t = targets[:live].long()
    has = t >= 0
    logprob = torch.where(has, ln.gather(1, t.clamp(min=0)[:, None])[:, 0], 0.0)
    entropy = torch.where(has, -(ln.exp() * ln).sum(1), 0.0)
    return (adv[:live].double() * logprob + ent[:live].double() * entropy).sum(), logprob, entropy


class Step:
    def __init__(self):
        self.cu = [int(v) for v in R.bounds_of(LENS)]
        self.live, T = self.cu[-1], self.cu[-1] + TAIL
        self.T = T
        g = torch.Generator().manual_seed(3)
        t = torch.randint(0, V, (T,), generator=g, dtype=torch.int32)
        t[torch.rand(T, generator=g) < 0.4] = -1  # prompts
        t[self.live:] = -1
        self.targets = t.cuda()
        self.adv = (torch.randn(T, generator=g) / T).cuda()
        self.ent = torch.full((T,), 0.01 / T, device="cuda")
        self.w = dict(embed=bf16_randn((V, H), 1, 0.1), wqkv=bf16_randn(((NQ + 2 * NKV) * D, H), 2, 0.06),
                      wo=bf16_randn((H, NQ * D), 3, 0.06), gq=bf16_randn((D,), 4, 0.1) + 1, gk=bf16_randn((D,), 5, 0.1) + 1,
                      g2=bf16_randn((H,), 6, 0.1) + 1)
        self.x = bf16_randn((T, H), 7)

        def new(*s, dt=BF16):
            return torch.zeros(*s, dtype=dt, device="cuda")

        def space(n):
            return torch.empty(n, dtype=torch.uint8, device="cuda")

        self.c, self.score = PackedConfig(T, len(LENS), NQ, NKV, D), ScoreConfig(cap=CAP, window=WINDOW)
        self.plan, self.bounds = space(L.ls_packed_plan_bytes(self.c)), torch.tensor(self.cu, dtype=torch.int32, device="cuda")
        n = (NQ + 2 * NKV) * D
        self.qkv, self.y, self.dqkv, self.dy = new(T, n), new(T, n), new(T, n), new(T, n)
        self.o, self.rest, self.do, self.lse = new(T, NQ * D), new(T, NQ * D), new(T, NQ * D), new(NQ, T, dt=F32)
        self.proj, self.h2, self.dh2, self.dx2, self.dx = (new(T, H) for _ in range(5))
        self.r2, self.logprob, self.entropy, self.hlse = (new(T, dt=F32) for _ in range(4))
        self.d = dict(embed=new(V, H, dt=F32), wqkv=new(n, H, dt=F32), wo=new(H, NQ * D, dt=F32), gq=new(D, dt=F32),
                      gk=new(D, dt=F32), g2=new(H, dt=F32))
        self.clipped = {k: torch.zeros_like(t, dtype=BF16) for k, t in self.d.items()}
        self.norm = new(1, dt=F32)
        self.ws = dict(head=space(L.ls_token_logprob_workspace(T, H, V)), norm=space(L.ls_rmsnorm_bwd_workspace(T, H)),
                       attn=space(L.ls_packed_attn_bwd_workspace(self.c)),
                       qk=space(L.ls_packed_qk_norm_rope_bwd_workspace(self.c)), grad=space(L.ls_grad_norm_workspace()))

    def run(self, max_norm):
        w, d, ws, c, T, live = self.w, self.d, self.ws, self.c, self.T, self.live
        L.ls_packed_plan(c, self.bounds, self.plan)
        L.ls_gemm_nt(self.x, w["wqkv"], self.qkv)
        L.ls_packed_qk_norm_rope(c, self.plan, THETA, EPS, w["gq"], w["gk"], self.qkv, self.y)
        L.ls_packed_score_attn_fwd(c, self.score, self.plan, self.y, self.o, self.lse, o_rest=self.rest)
        L.ls_gemm_nt(self.o, w["wo"], self.proj)
        x2 = self.x + self.proj
        L.ls_rmsnorm_fwd(T, H, EPS, x2, w["g2"], self.h2, self.r2)
        L.ls_token_logprob_fwd(self.h2, w["embed"], self.targets, self.logprob, self.entropy, self.hlse, ws["head"], scale=SCALE)
        L.ls_token_logprob_bwd(self.h2, w["embed"], self.targets, self.entropy, self.hlse, self.adv, self.ent, self.dh2,
                               d["embed"], False, ws["head"], scale=SCALE)
        L.ls_rmsnorm_bwd(T, H, x2, w["g2"], self.r2, self.dh2, None, self.dx2, d["g2"], False, ws["norm"])
        L.ls_gemm_nn(self.dx2, w["wo"], self.do)
        L.ls_gemm_tn(self.dx2, self.o, d["wo"])
        L.ls_packed_score_attn_bwd(c, self.score, self.plan, self.y, self.o, self.lse, self.do, self.dy, ws["attn"],
                                   o_rest=self.rest)
        L.ls_packed_qk_norm_rope_bwd(c, self.plan, THETA, EPS, w["gq"], w["gk"], self.qkv, self.dy, self.dqkv, d["gq"], d["gk"],
                                     False, ws["qk"])
        L.ls_gemm_tn(self.dqkv, self.x, d["wqkv"])
        L.ls_grad_norm(list(d.values()), self.norm, ws["grad"])
        L.ls_grad_clip(list(d.values()), self.norm, max_norm, list(self.clipped.values()))
        return self

    def results(self):
        return [self.logprob, self.entropy, self.norm, *self.d.values(), *self.clipped.values()]


def test_step():
    need_gpu()
    s = Step().run(1e-3)
    w64 = {k: t.double().requires_grad_() for k, t in s.w.items()}
    loss, logprob, entropy = model64(s.x.double(), s.targets, s.adv, s.ent, w64, s.cu)
    loss.backward()
    for name, got, ref in (("logprob", s.logprob, logprob), ("entropy", s.entropy, entropy)):
        err = float((got[:s.live].double() - ref).abs().max() / ref.abs().max())
        say(f"{name}: {err:.2e}")
        assert err <= OUT_TOL
        assert not got[s.live:].any()
    total = torch.sqrt(sum(t.grad.pow(2).sum() for t in w64.values()))
    say(f"norm {s.norm.item():.6f} against {total.item():.6f}")
    assert abs(s.norm.item() - total.item()) <= GRAD_TOL * total.item()
    assert s.norm.item() > 2e-3  # clipped in earnest
    for k, t in w64.items():
        rel = float((s.d[k].double() - t.grad).norm() / t.grad.norm())
        say(f"{k}: {rel:.2e}")
        assert rel <= GRAD_TOL, k
        want = s.d[k].double() * (1e-3 / (s.norm.double() + 1e-6))
        assert bool(((s.clipped[k].double() - want).abs() <= (2.0 ** -8 + 2.0 ** -22) * want.abs() + 1e-37).all()), k


def test_captured_step():
    """Replays after eager steps on other data, every one against the eager result."""
    need_gpu()
    s = Step()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        s.run(1e-3)
    torch.cuda.current_stream().wait_stream(side)
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        s.run(1e-3)
    for i in range(3):
        s.x.copy_(bf16_randn(s.x.shape, 50 + i))
        s.targets[:s.live].copy_(torch.roll(s.targets[:s.live], 5))
        s.bounds.copy_(torch.tensor([0, 10 * i, 100, 100, 101, 200, 280, s.live], dtype=torch.int32))
        s.run(1e-3)
        torch.cuda.synchronize()
        want = [t.clone() for t in s.results()]
        for t in s.results():
            t.fill_(3.0)
        g.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(want, s.results()))
