"""q/k norm with rotation on packed sequences, forward and backward, against the 64-bit reference of score_ref."""
from __future__ import annotations

import numpy as np
import pytest
import torch

import score_ref as S
from gpu_util import bf16_randn, f64, need_gpu, say
from paper_2510_02483_amd import lib as L
from paper_2510_02483_amd.configs import PackedConfig
from test_gpu_packed import LENGTHS, MARK, Batch

pytestmark = pytest.mark.gpu
EPS = 1e-5
HEADS = [(4, 2, 64), (24, 8, 128), (3, 3, 128), (7, 7, 104), (5, 1, 72), (2, 1, 80), (1, 1, 88), (17, 1, 112), (8, 1, 120), (33, 3, 96)]


class Norm:
    """A batch with gains and the gradient of every row, and the calls on it."""

    def __init__(self, b, theta=5e5, eps=EPS, seed=50):
        self.b, self.theta, self.eps, c = b, theta, eps, b.c
        self.gq, self.gk = ((1.0 + 0.3 * bf16_randn((b.d,), seed + i).float()).to(torch.bfloat16) for i in (0, 1))
        self.dy = bf16_randn(b.qkv.shape, seed + 2)
        self.dy[b.outside] = float("nan")
        self.y, self.dx = torch.full_like(b.qkv, MARK), torch.full_like(b.qkv, MARK)
        self.dgq, self.dgk = (torch.full((b.d,), MARK, device="cuda") for _ in range(2))
        self.ws = torch.empty(L.ls_packed_qk_norm_rope_bwd_workspace(c), dtype=torch.uint8, device="cuda")
        L.ls_packed_plan(c, b.cu, b.plan)

    def fwd(self, src=None, dst=None):
        b = self.b
        L.ls_packed_qk_norm_rope(b.c, b.plan, self.theta, self.eps, self.gq, self.gk, b.qkv if src is None else src,
                                 self.y if dst is None else dst)
        return self

    def bwd(self, dy=None, dx=None, dgq=0, dgk=0, accumulate=False):
        b = self.b
        L.ls_packed_qk_norm_rope_bwd(b.c, b.plan, self.theta, self.eps, self.gq, self.gk, b.qkv,
                                     self.dy if dy is None else dy, self.dx if dx is None else dx,
                                     self.dgq if dgq == 0 else dgq, self.dgk if dgk == 0 else dgk, accumulate, self.ws)
        return self

    def want(self):
        x, _ = self.b.inputs64()
        dy = f64(self.dy)
        dy[self.b.outside.cpu().numpy()] = 0.0
        b = self.b
        return S.qk_norm_rope(x, b.lens, b.first, b.nq, b.nkv, b.d, self.theta, self.eps, f64(self.gq), f64(self.gk), dy)

    def check(self):
        out = self.b.outside.cpu().numpy()
        v = (self.b.nq + self.b.nkv) * self.b.d
        want = self.want()
        for name, got, (ref, lim) in zip(("y", "dx", "dgq", "dgk"), (self.y, self.dx, self.dgq, self.dgk), want):
            got = f64(got)
            if got.ndim == 2:
                assert np.all(got[out] == MARK), name
                assert np.all(got[~out][:, v:] == ref[~out][:, v:]), f"{name}: v is copied"
                got, ref, lim = got[~out][:, :v], ref[~out][:, :v], lim[~out][:, :v]
            err = np.abs(got - ref)
            assert np.all(err <= lim), (name, float(np.max(err / lim)))
            if err.size:
                say(f"{name}: worst share of the bound {np.max(err / np.maximum(lim, 1e-300)):.2f}")


@pytest.mark.parametrize("nq,nkv,d", HEADS)
@pytest.mark.parametrize("lens", LENGTHS, ids=list(LENGTHS))
def test_against_the_reference(lens, nq, nkv, d):
    need_gpu()
    say(lens, nq, nkv, d)
    Norm(Batch(nq=nq, nkv=nkv, d=d, seed=11, **LENGTHS[lens])).fwd().bwd().check()


@pytest.mark.parametrize("nq,nkv,d", [(16, 2, 128), (32, 8, 64), (64, 64, 104), (48, 3, 72), (32, 1, 88), (128, 4, 64)])
@pytest.mark.parametrize("lens", ["one_row", "empty_ones", "mixed"])
def test_rows_that_several_waves_share(lens, nq, nkv, d):
    """Heads that are cut evenly, with key heads that are not, in place too."""
    need_gpu()
    n = Norm(Batch(nq=nq, nkv=nkv, d=d, seed=13, **LENGTHS[lens])).fwd().bwd()
    n.check()
    inside = ~n.b.outside
    work = n.b.qkv.clone()
    n.fwd(work, work)
    assert torch.equal(work[inside], n.y[inside]) and torch.isnan(work[~inside]).all()
    work, gains = n.dy.clone(), (n.dgq.clone(), n.dgk.clone())
    n.bwd(work, work)
    assert torch.equal(work[inside], n.dx[inside]) and torch.isnan(work[~inside]).all()
    assert torch.equal(gains[0], n.dgq) and torch.equal(gains[1], n.dgk)


@pytest.mark.parametrize("total", [16383, 32767, 32768])
def test_rows_around_the_number_that_is_cut(total):
    need_gpu()
    Norm(Batch([total - 5, 1, 4], 16, 1, 64 + 8, seed=14)).fwd().bwd().check()


@pytest.mark.parametrize("nq,nkv,d", [(4, 2, 64), (2, 1, 104)])
def test_many_rows(nq, nkv, d):
    """More rows than the backward pass has waves."""
    need_gpu()
    Norm(Batch([3000, 1, 0, 7000], nq, nkv, d, first=1, tail=3, seed=12)).fwd().bwd().check()


@pytest.mark.parametrize("nq,nkv,d", [(4, 2, 64), (3, 1, 128), (6, 2, 72)])
def test_in_place(nq, nkv, d):
    need_gpu()
    n = Norm(Batch([50, 0, 1, 333], nq, nkv, d, first=2, tail=5, seed=11)).fwd().bwd()
    inside = ~n.b.outside
    work = n.b.qkv.clone()
    n.fwd(work, work)
    assert torch.equal(work[inside], n.y[inside]) and torch.isnan(work[~inside]).all()
    work = n.dy.clone()
    gains = n.dgq.clone(), n.dgk.clone()
    n.bwd(work, work)
    assert torch.equal(work[inside], n.dx[inside]) and torch.isnan(work[~inside]).all()
    assert torch.equal(gains[0], n.dgq) and torch.equal(gains[1], n.dgk)


def test_gains_that_are_frozen_or_added_to():
    need_gpu()
    n = Norm(Batch([50, 0, 1, 333], 4, 2, 64, seed=11)).bwd()
    dx, dgq, dgk = n.dx.clone(), n.dgq.clone(), n.dgk.clone()
    n.dgq.fill_(3.0), n.dgk.fill_(-2.0)
    n.bwd(accumulate=True)
    # (added in 64 bits, rounded once)
    assert torch.allclose(n.dgq, dgq + 3.0, rtol=2.0 ** -22, atol=2.0 ** -22) and \
        torch.allclose(n.dgk, dgk - 2.0, rtol=2.0 ** -22, atol=2.0 ** -22)
    for q, k in ((None, 0), (0, None), (None, None)):
        n.dgq.fill_(MARK), n.dgk.fill_(MARK), n.dx.fill_(MARK)
        n.bwd(dgq=q, dgk=k)
        assert torch.equal(n.dx, dx)
        assert torch.equal(n.dgq, dgq if q == 0 else torch.full_like(dgq, MARK))
        assert torch.equal(n.dgk, dgk if k == 0 else torch.full_like(dgk, MARK))


def test_no_row_of_a_sequence():
    need_gpu()
    n = Norm(Batch([0, 0], 4, 2, 64, first=3, tail=140, seed=11)).fwd().bwd()
    assert not n.dgq.any() and not n.dgk.any()


@pytest.mark.parametrize("nq,nkv,d", [(3, 1, 128), (5, 1, 72)])
def test_eps_of_zero_and_sizes_far_from_one(nq, nkv, d):
    """Lanes without a head, whose squares are 0, add nothing; rows of 1e-15 and 1e15."""
    need_gpu()
    n = Norm(Batch([40, 9], nq, nkv, d, seed=13), eps=0.0)
    n.b.qkv[::3] *= 1e15
    n.b.qkv[1::3] *= 1e-15
    n.fwd().bwd()
    n.check()


def test_a_head_of_zeros():
    need_gpu()
    n = Norm(Batch([40, 9], 3, 1, 64, seed=13))
    n.b.qkv[5, :64] = 0.0
    n.fwd().bwd().check()
    assert not n.y[5, :64].any()


def test_far_positions():
    need_gpu()
    rows = 200_003
    n = Norm(Batch([3, rows], 1, 1, 64, seed=13), theta=1e4).fwd()
    pick = np.r_[3 + 65536, 3 + 131072, rows - 5:rows + 3]
    x = f64(n.b.qkv)[pick]
    ang = np.outer(pick - 3, 1e4 ** (-2.0 * np.arange(32) / 64))
    got = f64(n.y)[pick]
    for h, g in enumerate((f64(n.gq), f64(n.gk))):
        v = x[:, 64 * h:64 * h + 64]
        v = v / np.sqrt((v * v).mean(1, keepdims=True) + EPS) * g
        lo, hi = v[:, :32], v[:, 32:]
        ref = np.concatenate([lo * np.cos(ang) - hi * np.sin(ang), lo * np.sin(ang) + hi * np.cos(ang)], 1)
        size = np.concatenate([np.abs(lo) + np.abs(hi)] * 2, 1)
        assert np.all(np.abs(got[:, 64 * h:64 * h + 64] - ref) <= 2.0 ** -8 * np.abs(ref) * 1.01 + 2.0 ** -17 * size)


def test_gradient_against_differences():
    need_gpu()
    b = Batch([20, 3], 2, 1, 64, seed=17)
    n = Norm(b).bwd()
    x, dy = f64(b.qkv), f64(n.dy)
    rng = np.random.default_rng(1)

    def loss(x, gq, gk):
        return (S.qk_norm_rope(x, b.lens, 0, 2, 1, 64, n.theta, EPS, gq, gk)[0] * dy).sum()

    gq, gk = f64(n.gq), f64(n.gk)
    sx, sq, sk = (rng.standard_normal(t.shape) for t in (x, gq, gk))
    diff = (loss(x + 1e-6 * sx, gq, gk) - loss(x - 1e-6 * sx, gq, gk)) / 2e-6
    got = f64(n.dx)
    # one rounding of every entry, in a random direction: five standard deviations
    assert abs((got * sx).sum() - diff) < 5 * 2.0 ** -8 * np.linalg.norm(got) + 1e-4 * abs(diff)
    diff = (loss(x, gq + 1e-6 * sq, gk + 1e-6 * sk) - loss(x, gq - 1e-6 * sq, gk - 1e-6 * sk)) / 2e-6
    assert abs((f64(n.dgq) * sq).sum() + (f64(n.dgk) * sk).sum() - diff) < 1e-4 * np.linalg.norm(f64(n.dgq)) * 8


def test_offsets_past_32_bits():
    """A buffer of more than 4 GiB: its last rows."""
    need_gpu()
    nq, nkv, d, rows = 64, 16, 128, 180_000
    c = PackedConfig(rows, 2, nq, nkv, d)
    qkv = torch.empty(rows, (nq + 2 * nkv) * d, dtype=torch.bfloat16, device="cuda")
    assert qkv.numel() * 2 > 1 << 32
    tail = bf16_randn((70, qkv.shape[1]), 3)
    qkv[-70:] = tail
    cu = torch.tensor([0, rows - 70, rows], dtype=torch.int32, device="cuda")
    qkv[:-70] = 1.0
    plan = torch.empty(L.ls_packed_plan_bytes(c), dtype=torch.uint8, device="cuda")
    L.ls_packed_plan(c, cu, plan)
    small = Norm(Batch([70], nq, nkv, d, seed=1))
    small.b.qkv, small.dy = tail, bf16_randn(tail.shape, 4)
    small.fwd().bwd()
    L.ls_packed_qk_norm_rope(c, plan, small.theta, EPS, small.gq, small.gk, qkv, qkv)
    assert torch.equal(qkv[-70:], small.y)
    del plan
    qkv[-70:] = tail
    plan = torch.empty(L.ls_packed_plan_bytes(c), dtype=torch.uint8, device="cuda")
    L.ls_packed_plan(c, cu, plan)
    dy = torch.zeros_like(qkv)
    dy[-70:] = small.dy
    ws = torch.empty(L.ls_packed_qk_norm_rope_bwd_workspace(c), dtype=torch.uint8, device="cuda")
    L.ls_packed_qk_norm_rope_bwd(c, plan, small.theta, EPS, small.gq, small.gk, qkv, dy, dy, small.dgq, small.dgk,
                                 False, ws)
    assert torch.equal(dy[-70:], small.dx) and not dy[:1000].any()


def test_replays():
    need_gpu()
    n = Norm(Batch([90, 40, 300, 17], 4, 2, 104, seed=9, tail=20)).fwd().bwd()
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        n.fwd().bwd()
    for lens in ([5, 260, 0, 182], [447, 0, 0, 0], [90, 40, 300, 17]):
        other = Batch(lens, 4, 2, 104, seed=9, tail=20)
        want = Norm(other).fwd().bwd()
        n.b.cu.copy_(other.cu)
        L.ls_packed_plan(n.b.c, n.b.cu, n.b.plan)
        for t in (n.y, n.dx, n.dgq, n.dgk):
            t.fill_(MARK)
        torch.cuda.synchronize()
        g.replay()
        torch.cuda.synchronize()
        for a, b in ((n.y, want.y), (n.dx, want.dx), (n.dgq, want.dgq), (n.dgk, want.dgk)):
            assert torch.equal(a, b)
