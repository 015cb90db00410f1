"""Packed attention with capped scores and windows on the GPU against the 64-bit reference of score_ref."""
from __future__ import annotations

import numpy as np
import pytest
import torch

import score_ref as S
from gpu_util import f64, need_gpu, say
from paper_2510_02483_amd import lib as L
from paper_2510_02483_amd.configs import PackedConfig, ScoreConfig
from test_gpu_packed import LENGTHS, MARK, Batch

pytestmark = pytest.mark.gpu


def run(b, score, backward=True, stream=None, rest=False):
    b.rest = torch.full_like(b.o, MARK) if rest else None
    L.ls_packed_plan(b.c, b.cu, b.plan, stream=stream)
    L.ls_packed_score_attn_fwd(b.c, score, b.plan, b.qkv, b.o, b.lse, o_rest=b.rest, stream=stream)
    if backward:
        L.ls_packed_score_attn_bwd(b.c, score, b.plan, b.qkv, b.o, b.lse, b.dout, b.dqkv, b.ws, o_rest=b.rest,
                                   stream=stream)
    return b


def check(b, score, backward=True):
    x, g = b.inputs64()
    rest = b.rest is not None
    o, lse, grad, tol = S.attention(x, b.lens, b.first, b.nq, b.nkv, b.d, g, score.scale, score.cap, score.window, rest)
    out = b.outside.cpu().numpy()
    if rest:
        assert np.all(f64(b.rest)[out] == MARK)
        # o and its rest: the rounding of p is left, and two of fp32
        lim = tol["o"] - S.U * np.abs(o) * 1.01 + 2.0 ** -16 * np.abs(o) + 1e-30
        assert np.all(np.abs(f64(b.o) + f64(b.rest) - o)[~out] <= lim[~out])
        assert np.all(np.abs(f64(b.rest)[~out]) <= S.U * np.abs(f64(b.o)[~out]))
    pairs = [("o", f64(b.o), o, tol["o"]), ("lse", f64(b.lse).T, lse.T, tol["lse"].T)]
    if backward:
        pairs.append(("dqkv", f64(b.dqkv), grad, tol["dqkv"]))
    for name, got, ref, lim in pairs:
        assert np.all(got[out] == MARK), f"{name}: rows of no sequence written"
        err = np.abs(got[~out] - ref[~out])
        assert np.all(err <= lim[~out]), (name, float(np.max(err / lim[~out])))
        if not out.all():
            say(f"{name}: rel {np.linalg.norm(err) / max(np.linalg.norm(ref[~out]), 1e-300):.2e}, "
                f"worst share of the bound {np.max(err / lim[~out]):.2f}")


SCORES = {
    "cap": ScoreConfig(cap=10.0),
    "cap_scale": ScoreConfig(scale=0.3, cap=50.0),
    "wide_cap": ScoreConfig(cap=300.0),
    "window": ScoreConfig(window=37),
    "window_of_one": ScoreConfig(window=1),
    "window_of_a_tile": ScoreConfig(window=128),
    "cap_window": ScoreConfig(cap=20.0, window=70),
    "scale": ScoreConfig(scale=0.05),
}


@pytest.mark.parametrize("nq,nkv,d", [(4, 2, 64), (3, 1, 128), (4, 2, 104)])
@pytest.mark.parametrize("score", SCORES, ids=list(SCORES))
@pytest.mark.parametrize("lens", LENGTHS, ids=list(LENGTHS))
def test_against_the_reference(lens, score, nq, nkv, d):
    need_gpu()
    say(lens, score, nq, nkv, d)
    for rest in (False, True):
        b = Batch(nq=nq, nkv=nkv, d=d, seed=3, std=2.0, **LENGTHS[lens])
        check(run(b, SCORES[score], rest=rest), SCORES[score])


@pytest.mark.parametrize("nq,nkv,d", [(4, 2, 64), (8, 1, 128), (5, 1, 120)])
@pytest.mark.parametrize("window", [1, 65, 300, 1000, 2499])
def test_a_long_sequence_through_a_window(window, nq, nkv, d):
    """The plan cuts the work of the first keys into parts that a window leaves few steps or none."""
    need_gpu()
    score = ScoreConfig(cap=15.0 if window in (65, 1000) else 0.0, window=window)
    check(run(Batch([40, 2500, 3, 100], nq, nkv, d, tail=2, seed=27, std=1.5), score), score)


@pytest.mark.parametrize("nq,nkv,d", [(7, 1, 64), (8, 1, 128)])
@pytest.mark.parametrize("score", [ScoreConfig(cap=5.0), ScoreConfig(window=9), ScoreConfig(cap=30.0, window=33)],
                         ids=["cap", "window", "both"])
def test_many_small_sequences_of_a_group(score, nq, nkv, d):
    need_gpu()
    lens = [1, 32, 33, 64, 0, 17, 50] * 12
    check(run(Batch(lens + [65, 140], nq, nkv, d, tail=5, seed=35, std=2.0), score), score)


@pytest.mark.parametrize("lens", [[1], [64], [33, 2], [20, 64, 0, 7]])
@pytest.mark.parametrize("nq,nkv,d", [(32, 2, 64), (16, 1, 128)])
def test_few_small_sequences_of_a_large_group(lens, nq, nkv, d):
    need_gpu()
    score = ScoreConfig(cap=8.0, window=21)
    check(run(Batch(lens, nq, nkv, d, first=1, tail=2, seed=37, std=2.0), score), score)


def test_the_rest_of_o_alone():
    """Plain scores with a rest: o and lse within their bounds, the gradients nearer than the plain attention's."""
    need_gpu()
    a, b = (Batch([600, 90, 20], 4, 2, 64, tail=3, seed=9, std=2.0) for _ in range(2))
    a.run()
    run(b, ScoreConfig(), rest=True)
    check(b, ScoreConfig())
    x, g = a.inputs64()
    ref = S.attention(x, a.lens, 0, 4, 2, 64, g)[2]
    off = [np.linalg.norm((f64(t.dqkv) - ref)[:710]) for t in (a, b)]
    assert off[1] < off[0]


@pytest.mark.parametrize("cap", [0.01, 1.0, 30.0, 50.0, 60.0, 1000.0])
@pytest.mark.parametrize("d", [64, 128])
def test_scores_far_beyond_the_cap(d, cap):
    """Scores of several hundreds of either sign: the cap's ends, where its slope vanishes."""
    need_gpu()
    score = ScoreConfig(cap=cap)
    check(run(Batch([200, 70, 30, 5], 2, 1, d, seed=5, std=8.0), score), score)


@pytest.mark.parametrize("sign", [1.0, -1.0])
def test_all_scores_at_one_end_of_the_cap(sign):
    """Every score of a row at +cap or -cap: the softmax is flat, whatever the reference of its exponents."""
    need_gpu()
    for cap in (20.0, 50.0, 1000.0):
        b = Batch([150, 40, 9], 2, 1, 128, seed=6, std=1.0)
        b.qkv[:, :2 * 128], b.qkv[:, 2 * 128:3 * 128] = 16.0, sign * 16.0
        b.qkv[b.outside] = float("nan")
        run(b, ScoreConfig(cap=cap))
        check(b, ScoreConfig(cap=cap))
        if cap < 100.0:  # (scores of 2896)
            assert torch.allclose(b.lse[:, 0], torch.full_like(b.lse[:, 0], sign * cap), rtol=1e-5)


@pytest.mark.parametrize("window", [0, 400, 10_000])
def test_without_a_cap_and_all_in_the_window_is_the_plain_attention(window):
    need_gpu()
    a, b = (Batch([90, 40, 300, 17], 4, 2, 64, tail=3, seed=9) for _ in range(2))
    a.run()
    run(b, ScoreConfig(window=450 if window == 400 else window))
    for x, y in ((a.o, b.o), (a.lse, b.lse), (a.dqkv, b.dqkv)):
        assert torch.equal(x, y)


def test_a_cap_far_above_the_scores_changes_little():
    need_gpu()
    a, b = (Batch([90, 40, 300, 17], 4, 2, 64, seed=9, std=0.5) for _ in range(2))
    a.run()
    run(b, ScoreConfig(cap=1000.0))
    # x - tanh x < x^3 / 3: scores of at most 3 differ by 1e-5; the capped ones are good to 1000 x 2^-21
    assert (a.lse - b.lse).abs().max() < 1e-3
    assert (a.o.float() - b.o.float()).abs().max() <= 2.0 ** -7


def test_neighbours_do_not_matter():
    need_gpu()
    score = ScoreConfig(cap=10.0, window=60)
    lens = [90, 40, 300, 17]
    a = run(Batch(lens, 4, 2, 64, seed=9), score)
    b = Batch(lens, 4, 2, 64, seed=9)
    b.qkv[90:130] = float("nan")
    b.dout[90:130] = float("inf")
    b.qkv[430:] = float("-inf")
    run(b, score)
    for rows in (slice(0, 90), slice(130, 430)):
        assert torch.equal(a.o[rows], b.o[rows]) and torch.equal(a.lse[:, rows], b.lse[:, rows])
        assert torch.equal(a.dqkv[rows], b.dqkv[rows])
    assert torch.isnan(b.o[90:130]).all()


@pytest.mark.parametrize("nq,nkv,d", [(6, 2, 64), (6, 3, 128)])
def test_backward_in_one_launch_or_two(nq, nkv, d):
    need_gpu()
    score = ScoreConfig(cap=12.0, window=150)
    lens = [40, 500, 3, 100, 230, 64, 31]
    few = run(Batch(lens, nq, nkv, d, tail=1, seed=31), score)
    many = Batch(lens, nq, nkv, d, tail=22_000, seed=31)
    rows = sum(lens)
    many.qkv[:rows], many.dout[:rows] = few.qkv[:rows], few.dout[:rows]
    run(many, score)
    for a, b in ((few.o, many.o), (few.dqkv[:, :nq * d], many.dqkv[:, :nq * d])):
        assert torch.equal(a[:rows], b[:rows])
        assert (b[rows:] == MARK).all()
    few.dqkv = many.dqkv[:rows + 1]
    check(few, score)


def test_differences_of_the_loss():
    """The gradient against differences of sum(o dout), taken in 64 bits from the reference's forward pass."""
    need_gpu()
    b = run(Batch([37, 90], 2, 1, 64, seed=41, std=1.5), ScoreConfig(cap=6.0, window=40))
    x, g = b.inputs64()
    rng = np.random.default_rng(0)
    for _ in range(4):
        step = rng.standard_normal(x.shape)
        f = [(S.attention(x + t * step, b.lens, 0, 2, 1, 64, None, 0.0, 6.0, 40)[0] * g).sum() for t in (1e-5, -1e-5)]
        got = (f64(b.dqkv) * step).sum()
        # the gradient is off by two or three roundings (2^-8 each) of every entry, which a random direction averages
        assert abs(got - (f[0] - f[1]) / 2e-5) < 8 * 2.0 ** -8 * np.linalg.norm(f64(b.dqkv)) + 1e-6


def test_replays_with_other_lengths_and_two_streams():
    need_gpu()
    score = ScoreConfig(cap=9.0, window=50)
    first, other = [90, 40, 300, 17], [5, 260, 0, 182]
    b = Batch(first, 4, 2, 64, seed=9)
    run(b, score)
    g = torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    with torch.cuda.graph(g):
        run(b, score)
    for lens in (other, first, other):
        want = run(Batch(lens, 4, 2, 64, seed=9), score)
        b.cu.copy_(want.cu)
        b.o.fill_(MARK), b.lse.fill_(MARK), b.dqkv.fill_(MARK)
        torch.cuda.synchronize()
        g.replay()
        torch.cuda.synchronize()
        assert torch.equal(b.o, want.o) and torch.equal(b.lse, want.lse) and torch.equal(b.dqkv, want.dqkv)
    batches = [Batch([700, 33, 9], 4, 2, 64, seed=s) for s in (1, 2)]
    scores = [score, ScoreConfig(window=128)]
    streams = [torch.cuda.Stream() for _ in batches]
    torch.cuda.synchronize()
    for x, sc, st in zip(batches, scores, streams):
        run(x, sc, stream=st)
    torch.cuda.synchronize()
    for x, sc in zip(batches, scores):
        check(x, sc)


def test_a_plan_of_garbage_leads_nowhere():
    """Whatever the plan holds, nothing outside the buffers is touched."""
    need_gpu()
    score = ScoreConfig(cap=9.0, window=50)
    b = Batch([300, 40], 4, 2, 64, seed=9)
    room = 1 << 16
    for value in (0, 0x7F, 0xFF, 0x11):
        b.plan.fill_(value)
        guarded = [torch.full((t.numel() + 2 * room,), 5.0, dtype=t.dtype, device="cuda") for t in (b.o, b.lse, b.dqkv)]
        o, lse, dqkv = (t[room:-room] for t in guarded)
        L.ls_packed_score_attn_fwd(b.c, score, b.plan, b.qkv, o, lse)
        L.ls_packed_score_attn_bwd(b.c, score, b.plan, b.qkv, b.o, b.lse, b.dout, dqkv, b.ws)
        torch.cuda.synchronize()
        for t in guarded:
            assert (t[:room] == 5.0).all() and (t[-room:] == 5.0).all()
