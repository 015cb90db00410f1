"""Packed sequences on the GPU against the 64-bit reference of packed_ref."""
from __future__ import annotations

import numpy as np
import pytest
import torch

import packed_ref as R
from gpu_util import bf16_randn, f64, need_gpu, say
from paper_2510_02483_amd import lib as L
from paper_2510_02483_amd.configs import B3, PackedConfig

pytestmark = pytest.mark.gpu

MARK = 77.0  # what outputs hold before a call


class Batch:
    """Random qkv and dout of one row of packed sequences; rows of none hold NaN."""

    def __init__(self, lens, nq, nkv, d, first=0, tail=0, seed=0, std=1.0):
        self.lens, self.first, self.nq, self.nkv, self.d = list(lens), first, nq, nkv, d
        self.total = first + sum(lens) + tail
        self.c = PackedConfig(self.total, len(lens), nq, nkv, d)
        self.cu = torch.tensor(R.bounds_of(lens, first), dtype=torch.int32, device="cuda")
        self.qkv = bf16_randn((self.total, (nq + 2 * nkv) * d), seed, std)
        self.dout = bf16_randn((self.total, nq * d), seed + 1)
        self.outside = torch.ones(self.total, dtype=torch.bool, device="cuda")
        self.outside[first:first + sum(lens)] = False
        self.qkv[self.outside] = float("nan")
        self.dout[self.outside] = float("nan")
        self.plan = torch.empty(L.ls_packed_plan_bytes(self.c), dtype=torch.uint8, device="cuda")
        self.o = torch.full((self.total, nq * d), MARK, dtype=torch.bfloat16, device="cuda")
        self.lse = torch.full((nq, self.total), MARK, dtype=torch.float32, device="cuda")
        self.dqkv = torch.full_like(self.qkv, MARK)
        self.ws = torch.empty(L.ls_packed_attn_bwd_workspace(self.c), dtype=torch.uint8, device="cuda")

    def run(self, backward=True, stream=None):
        L.ls_packed_plan(self.c, self.cu, self.plan, stream=stream)
        L.ls_packed_attn_fwd(self.c, self.plan, self.qkv, self.o, self.lse, stream=stream)
        if backward:
            L.ls_packed_attn_bwd(self.c, self.plan, self.qkv, self.o, self.lse, self.dout, self.dqkv, self.ws,
                                 stream=stream)
        return self

    def inputs64(self):
        x, g = f64(self.qkv), f64(self.dout)
        out = self.outside.cpu().numpy()
        x[out], g[out] = 0.0, 0.0
        return x, g


def check(b, backward=True):
    x, g = b.inputs64()
    o, lse, grad, tol = R.attention(x, b.lens, b.first, b.nq, b.nkv, b.d, g)
    out = b.outside.cpu().numpy()
    pairs = [("o", f64(b.o), o, ~out), ("lse", f64(b.lse).T, lse.T, ~out)]
    if backward:
        pairs.append(("dqkv", f64(b.dqkv), grad, ~out))
    for name, got, ref, rows in pairs:
        lim = tol[name].T if name == "lse" else tol[name]
        assert np.all(got[out] == MARK), f"{name}: rows of no sequence written"
        err = np.abs(got[rows] - ref[rows])
        assert np.all(err <= lim[rows]), (name, float(np.max(err / lim[rows])))
        if rows.any():
            say(f"{name}: rel {np.linalg.norm(err) / max(np.linalg.norm(ref[rows]), 1e-300):.2e}, "
                f"worst share of the bound {np.max(err / lim[rows]):.2f}")


LENGTHS = {
    "one_row": dict(lens=[1]),
    "rows_of_one": dict(lens=[1] * 70, tail=3),
    "empty_ones": dict(lens=[0, 5, 0, 0, 131, 0], first=7, tail=9),
    "around_a_tile": dict(lens=[127, 128, 129, 63, 64, 65]),
    "small_ones": dict(lens=[31, 32, 33, 34, 63, 64, 65, 40, 48, 2, 64]),
    "mixed": dict(lens=[300, 1, 0, 513, 33, 2], tail=130),
    "all_empty": dict(lens=[0, 0], first=3, tail=140),
}


@pytest.mark.parametrize("nq,nkv,d", [(4, 2, 64), (2, 2, 128), (6, 1, 64), (3, 1, 128), (4, 2, 104), (1, 1, 72)])
@pytest.mark.parametrize("lens", LENGTHS, ids=list(LENGTHS))
def test_attention_matches_the_reference(lens, nq, nkv, d):
    need_gpu()
    say(lens, nq, nkv, d)
    check(Batch(nq=nq, nkv=nkv, d=d, seed=3, **LENGTHS[lens]).run())


@pytest.mark.parametrize("nq,nkv,d", [(4, 2, 64), (7, 1, 64), (8, 1, 128), (3, 1, 104)])
def test_many_small_sequences_of_a_group(nq, nkv, d):
    """More sequences of up to 64 rows than are listed as tiles (64 / nkv): waves and pairs of waves go through the
    heads of the group."""
    need_gpu()
    lens = [1, 32, 33, 64, 0, 17, 50] * 12
    check(Batch(lens + [65, 140], nq, nkv, d, tail=5, seed=35).run())


@pytest.mark.parametrize("lens", [[1], [64], [33, 2], [20, 64, 0, 7]])
@pytest.mark.parametrize("nq,nkv,d", [(32, 2, 64), (16, 1, 128)])
def test_few_small_sequences_of_a_large_group(lens, nq, nkv, d):
    need_gpu()
    check(Batch(lens, nq, nkv, d, first=1, tail=2, seed=37).run())


@pytest.mark.parametrize("d", [64, 128])
def test_peaked_scores(d):
    """Scores up to a hundred: the running maximum moves, probabilities underflow."""
    need_gpu()
    b = Batch([200, 70], 2, 1, d, seed=5, std=4.0)
    L.ls_packed_plan(b.c, b.cu, b.plan)
    L.ls_packed_attn_fwd(b.c, b.plan, b.qkv, b.o, b.lse)
    x, _ = b.inputs64()
    o, lse, _, tol = R.attention(x, b.lens, 0, 2, 1, d)
    # the exponent s log2(e) - m at |s| up to 2^7 carries 2^-17 at most: 2^-16 relative on p instead of 2^-18
    assert np.all(np.abs(f64(b.o) - o) <= tol["o"] + 2.0 ** -15 * np.abs(x).max())
    assert np.all(np.abs(f64(b.lse) - lse) <= tol["lse"] + 2.0 ** -24 * 2 ** 8)


@pytest.mark.parametrize("nq,nkv,d", [(4, 2, 64), (3, 1, 128)])
def test_equal_lengths_are_the_attention_core(nq, nkv, d):
    """Sequences of one length give what ls_attn_core_fwd gives, bit for bit, and the dq of ls_attn_core_bwd; its
    dk and dv may be added in another order."""
    need_gpu()
    n, S = 3, 257
    b = Batch([S] * n, nq, nkv, d, seed=7).run()
    c = B3.with_(batch=n, seq=S, n_q_heads=nq, n_kv_heads=nkv, head_dim=d)
    o, lse = torch.empty_like(b.o), torch.empty(n, nq, S, device="cuda")
    L.ls_attn_core_fwd(c, b.qkv, o, lse)
    assert torch.equal(o, b.o)
    assert torch.equal(lse.permute(1, 0, 2).reshape(nq, -1), b.lse)
    dqkv = torch.empty_like(b.dqkv)
    ws = torch.empty(L.ls_attn_core_bwd_workspace(c), dtype=torch.uint8, device="cuda")
    L.ls_attn_core_bwd(c, b.qkv, o, lse, b.dout, dqkv, ws)
    assert torch.equal(dqkv[:, :nq * d], b.dqkv[:, :nq * d])
    check(b)


def test_neighbours_do_not_matter():
    """A sequence's results are the same bits whatever the others hold, NaN and infinities among it."""
    need_gpu()
    lens = [90, 40, 300, 17]
    a = Batch(lens, 4, 2, 64, seed=9).run()
    b = Batch(lens, 4, 2, 64, seed=9)
    b.qkv[90:130] = float("nan")
    b.dout[90:130] = float("inf")
    b.qkv[430:] = float("-inf")
    b.run()
    for rows in (slice(0, 90), slice(130, 430)):
        assert torch.equal(a.o[rows], b.o[rows]) and torch.equal(a.lse[:, rows], b.lse[:, rows])
        assert torch.equal(a.dqkv[rows], b.dqkv[rows])
    assert torch.isnan(b.o[90:130]).all()


@pytest.mark.parametrize("inverse", [False, True])
@pytest.mark.parametrize("nq,nkv,d", [(4, 2, 64), (24, 8, 128), (3, 3, 128), (7, 7, 104), (5, 1, 72), (2, 1, 80)])
def test_rope(nq, nkv, d, inverse):
    need_gpu()
    b = Batch([50, 0, 1, 333], nq, nkv, d, first=2, tail=5, seed=11)
    L.ls_packed_plan(b.c, b.cu, b.plan)
    dst = torch.full_like(b.qkv, MARK)
    L.ls_packed_rope(b.c, b.plan, 5e5, b.qkv, dst, inverse=inverse)
    x, _ = b.inputs64()
    ref = R.rope(x, b.lens, b.first, nq, nkv, d, 5e5, inverse)
    inside = ~b.outside.cpu().numpy()
    got = f64(dst)
    assert np.all(got[~inside] == MARK)
    # one rounding of the result; cos and sin of an angle good to 2^-22, four fp32 operations
    mag = np.abs(x).reshape(len(x), -1, 2, d // 2).sum(2, keepdims=True).repeat(2, 2).reshape(x.shape)
    assert np.all(np.abs(got - ref)[inside] <= (R.U * np.abs(ref) * 1.01 + 2.0 ** -21 * mag)[inside])
    assert torch.equal(dst[~b.outside][:, (nq + nkv) * d:], b.qkv[~b.outside][:, (nq + nkv) * d:])
    work = b.qkv.clone()
    L.ls_packed_rope(b.c, b.plan, 5e5, work, work, inverse=inverse)  # in place
    assert torch.equal(work[~b.outside], dst[~b.outside])
    assert torch.isnan(work[b.outside]).all()


def test_rope_far_positions():
    need_gpu()
    n = 200_003
    b = Batch([3, n], 1, 1, 64, seed=13)
    L.ls_packed_plan(b.c, b.cu, b.plan)
    dst = torch.empty_like(b.qkv)
    L.ls_packed_rope(b.c, b.plan, 1e4, b.qkv, dst)
    rows = np.r_[0:5, 3 + 65536, 3 + 131072, n - 5:n + 3]
    x = f64(b.qkv)[rows]
    pos = np.where(rows < 3, rows, rows - 3)
    ang = np.outer(pos, 1e4 ** (-2.0 * np.arange(32) / 64))
    got = f64(dst)[rows]
    for h in range(2):
        lo, hi = x[:, 64 * h:64 * h + 32], x[:, 64 * h + 32:64 * h + 64]
        ref = lo * np.cos(ang) - hi * np.sin(ang)
        assert np.all(np.abs(got[:, 64 * h:64 * h + 32] - ref) <= R.U * np.abs(ref) * 1.01 + 2.0 ** -21 * (abs(lo) + abs(hi)))


@pytest.mark.parametrize("nq,nkv,d", [(4, 2, 64), (2, 2, 128), (8, 1, 128), (5, 1, 120)])
def test_one_long_sequence_among_others(nq, nkv, d):
    """The dK/dV work of the long sequence's first keys is cut into parts."""
    need_gpu()
    check(Batch([40, 2500, 3, 100], nq, nkv, d, tail=2, seed=27).run())


@pytest.mark.parametrize("nq,nkv,d", [(6, 2, 64), (6, 3, 128), (6, 2, 88)])
def test_backward_in_one_launch_or_two(nq, nkv, d):
    """Rows behind the last sequence let the batch have more than 1024 query tiles times heads, the most whose dK/dV and
    dQ share a launch: the same bits."""
    need_gpu()
    lens = [40, 500, 3, 100, 230, 64, 31]
    few = Batch(lens, nq, nkv, d, tail=1, seed=31).run()
    many = Batch(lens, nq, nkv, d, tail=22_000, seed=31)
    rows = sum(lens)
    many.qkv[:rows], many.dout[:rows] = few.qkv[:rows], few.dout[:rows]
    many.run()
    for a, b in ((few.o, many.o), (few.dqkv, many.dqkv)):
        assert torch.equal(a[:rows], b[:rows])
        assert (b[rows:] == MARK).all()
    check(few)


@pytest.mark.parametrize("nq,nkv", [(1, 1), (2, 1)])
@pytest.mark.parametrize("total", [300_000, 3_000_000])
def test_short_sequences_in_a_long_row(total, nq, nkv):
    """A row so long that the plan keeps many ranks to a class: a tile's work is not cut into more parts than it has
    steps."""
    need_gpu()
    lens, d = [130, 65, 300, 1], 64
    small = Batch(lens, nq, nkv, d, seed=33).run()
    check(small)
    big = PackedConfig(total, len(lens), nq, nkv, d)
    plan = torch.empty(L.ls_packed_plan_bytes(big), dtype=torch.uint8, device="cuda")
    L.ls_packed_plan(big, small.cu, plan)
    rows = sum(lens)
    qkv, dout = (torch.zeros(total, x.shape[1], dtype=x.dtype, device="cuda") for x in (small.qkv, small.dout))
    qkv[:rows], dout[:rows] = small.qkv, small.dout
    o, dqkv, lse = torch.zeros_like(dout), torch.zeros_like(qkv), torch.zeros(nq, total, device="cuda")
    ws = torch.empty(L.ls_packed_attn_bwd_workspace(big), dtype=torch.uint8, device="cuda")
    L.ls_packed_attn_fwd(big, plan, qkv, o, lse)
    L.ls_packed_attn_bwd(big, plan, qkv, o, lse, dout, dqkv, ws)
    assert torch.equal(o[:rows], small.o) and torch.equal(dqkv[:rows, :nq * d], small.dqkv[:, :nq * d])
    small.dqkv = dqkv[:rows]
    check(small)
    assert not dqkv[rows:].any()


def test_many_sequences_and_every_row_once():
    """More sequences than the plan's workgroup has threads; the outputs do not depend on the order of its list."""
    need_gpu()
    rng = np.random.default_rng(3)
    lens = rng.integers(0, 12, 2500)
    lens[1234] = 1000
    b = Batch(lens, 1, 1, 64, tail=1, seed=15).run()
    check(b)
    again = Batch(lens, 1, 1, 64, tail=1, seed=15).run()
    assert torch.equal(b.dqkv, again.dqkv) and torch.equal(b.o, again.o)


def test_offsets_past_32_bits():
    """Sequences at the far end of buffers beyond 4 GiB give the bits they give in small ones."""
    need_gpu()
    lens, nq, nkv, d = [150, 65], 14, 2, 128
    total = 960_000  # x 18 x 128 x 2 = 4.4 GB of qkv
    small = Batch(lens, nq, nkv, d, seed=17).run()
    first = total - sum(lens)
    c = PackedConfig(total, len(lens), nq, nkv, d)
    cu = torch.tensor(R.bounds_of(lens, first), dtype=torch.int32, device="cuda")
    qkv = torch.zeros(total, (nq + 2 * nkv) * d, dtype=torch.bfloat16, device="cuda")
    dout = torch.zeros(total, nq * d, dtype=torch.bfloat16, device="cuda")
    qkv[first:], dout[first:] = small.qkv, small.dout
    plan = torch.empty(L.ls_packed_plan_bytes(c), dtype=torch.uint8, device="cuda")
    o, dqkv = torch.zeros_like(dout), torch.zeros_like(qkv)
    lse = torch.zeros(nq, total, device="cuda")
    L.ls_packed_plan(c, cu, plan)
    turned = qkv.clone()
    L.ls_packed_rope(c, plan, 1e4, turned, turned)
    L.ls_packed_attn_fwd(c, plan, qkv, o, lse)
    assert torch.equal(o[first:], small.o) and torch.equal(lse[:, first:], small.lse)
    assert not o[:first].any()
    ws = torch.empty(L.ls_packed_attn_bwd_workspace(c), dtype=torch.uint8, device="cuda")
    L.ls_packed_attn_bwd(c, plan, qkv, o, lse, dout, dqkv, ws)
    # dq is the same bits; dk and dv add the group's heads in one workgroup here, in seven there
    assert torch.equal(dqkv[first:, :nq * d], small.dqkv[:, :nq * d])
    torch.testing.assert_close(dqkv[first:].float(), small.dqkv.float(), rtol=2 * R.U, atol=2.0 ** -12)
    assert not dqkv[:first].any()
    sm = small.qkv.clone()
    L.ls_packed_rope(small.c, small.plan, 1e4, sm, sm)
    assert torch.equal(turned[first:], sm)


def test_lengths_out_of_order_stay_inside_the_buffers():
    """Entries that fall, that are negative or lie beyond the total, a plan that was never made or one of another
    shape: whatever comes out, nothing outside the outputs is written, and a good plan afterwards works."""
    need_gpu()
    b = Batch([100, 100, 100], 2, 1, 64, seed=19)
    b.plan = torch.empty(1 << 20, dtype=torch.uint8, device="cuda")
    pad = 4096
    for cu in ([0, 200, 100, 300], [-50, 100, 1000, 300], [300, 200, 100, 0], [0, 300, 0, 300], [2 ** 31 - 1, -2 ** 31, 5, 90],
               [0, 300, 300, 100], [10, 20, 15, 300], None, 0, 255, 1, PackedConfig(5000, 3, 2, 1, 64)):
        say(cu)
        flat = torch.full((b.dqkv.numel() + 2 * pad,), MARK, dtype=torch.bfloat16, device="cuda")
        of = torch.full((b.o.numel() + 2 * pad,), MARK, dtype=torch.bfloat16, device="cuda")
        dqkv, o = flat[pad:-pad].view_as(b.dqkv), of[pad:-pad].view_as(b.o)
        if cu is None:
            b.plan.random_(0, 256)
        elif isinstance(cu, int):
            b.plan.fill_(cu)
        elif isinstance(cu, PackedConfig):
            L.ls_packed_plan(cu, torch.tensor([0, 70, 200, 5000], dtype=torch.int32, device="cuda"), b.plan)
        else:
            L.ls_packed_plan(b.c, torch.tensor(cu, dtype=torch.int32, device="cuda"), b.plan)
        L.ls_packed_rope(b.c, b.plan, 1e4, b.qkv, dqkv)
        L.ls_packed_attn_fwd(b.c, b.plan, b.qkv, o, b.lse)
        L.ls_packed_attn_bwd(b.c, b.plan, b.qkv, o, b.lse, b.dout, dqkv, b.ws)
        torch.cuda.synchronize()
        for t in (flat, of):
            assert (t[:pad] == MARK).all() and (t[-pad:] == MARK).all()
    check(b.run())


def test_capture_replays_with_other_lengths():
    """A captured step reads the lengths that the buffer holds at the replay."""
    need_gpu()
    total, nq, nkv, d = 400, 4, 2, 64
    b = Batch([100, 250, 50], nq, nkv, d, seed=21)
    turned = torch.empty_like(b.qkv)
    grad = torch.empty_like(b.qkv)

    def step():
        L.ls_packed_plan(b.c, b.cu, b.plan)
        L.ls_packed_rope(b.c, b.plan, 1e4, b.qkv, turned)
        L.ls_packed_attn_fwd(b.c, b.plan, turned, b.o, b.lse)
        L.ls_packed_attn_bwd(b.c, b.plan, turned, b.o, b.lse, b.dout, b.dqkv, b.ws)
        L.ls_packed_rope(b.c, b.plan, 1e4, b.dqkv, grad, inverse=True)

    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        step()
    torch.cuda.current_stream().wait_stream(s)
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        step()
    for i, lens in enumerate(([100, 250, 50], [0, 1, 399], [133, 133, 134], [400, 0, 0])):
        b.cu.copy_(torch.tensor(R.bounds_of(lens), dtype=torch.int32))
        b.qkv.copy_(bf16_randn(b.qkv.shape, 100 + i))
        step()
        torch.cuda.synchronize()
        want = [t.clone() for t in (turned, b.o, b.lse, b.dqkv, grad)]
        for t in (turned, b.o, b.lse, b.dqkv, grad):
            t.zero_()
        g.replay()
        torch.cuda.synchronize()
        for t, w in zip((turned, b.o, b.lse, b.dqkv, grad), want):
            assert torch.equal(t, w), lens


def test_another_stream():
    need_gpu()
    a = Batch([30, 200], 4, 2, 64, seed=23).run()
    b = Batch([30, 200], 4, 2, 64, seed=23)
    torch.cuda.synchronize()
    s = torch.cuda.Stream()
    b.run(stream=s)
    s.synchronize()
    assert torch.equal(a.o, b.o) and torch.equal(a.dqkv, b.dqkv)


def test_two_streams_share_a_plan():
    """Layers on two streams at once: one plan, workspaces and outputs of their own."""
    need_gpu()
    lens = [700, 3, 60, 0, 400]
    a, b = Batch(lens, 8, 2, 64, seed=31), Batch(lens, 8, 2, 64, seed=33)
    want = [Batch(lens, 8, 2, 64, seed=s).run() for s in (31, 33)]
    L.ls_packed_plan(a.c, a.cu, a.plan)
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream(), torch.cuda.Stream()]
    for _ in range(5):
        for x, s in zip((a, b), streams):
            L.ls_packed_attn_fwd(x.c, a.plan, x.qkv, x.o, x.lse, stream=s)
            L.ls_packed_attn_bwd(x.c, a.plan, x.qkv, x.o, x.lse, x.dout, x.dqkv, x.ws, stream=s)
    torch.cuda.synchronize()
    for x, w in zip((a, b), want):
        assert torch.equal(x.o, w.o) and torch.equal(x.dqkv, w.dqkv)


def test_gradient_against_differences():
    """The kernels' gradient along a direction against the change of <dout, o> in 64 bits over the kernels' own
    rounded inputs."""
    need_gpu()
    b = Batch([40, 7, 90], 4, 2, 64, seed=25).run()
    x, g = b.inputs64()
    u = np.random.default_rng(5).standard_normal(x.shape)
    h = 1e-5
    up = (R.attention(x + h * u, b.lens, 0, 4, 2, 64)[0] * g).sum()
    down = (R.attention(x - h * u, b.lens, 0, 4, 2, 64)[0] * g).sum()
    tol = R.attention(x, b.lens, 0, 4, 2, 64, g)[3]["dqkv"]
    assert abs((f64(b.dqkv) * u).sum() - (up - down) / (2 * h)) <= (tol * np.abs(u)).sum() + 1e-5
