"""The head loss on the GPU against its definition in 64 bits.

Bounds count roundings: U = 2^-8 one rounding to bf16, W = 2^-24 one fp32 operation.  A logit is an fp32 sum of H
products: |err z| <= H W sum |h e|.  The log-sum-exp adds the exponent's rounding (at |z| log2(e) < 2^6: 2^-18
relative on a term), sums of V terms in blocks, and a logarithm."""
from __future__ import annotations

import pytest
import torch

from gpu_util import bf16_randn, need_gpu, say
from paper_2510_02483_amd import lib as L

pytestmark = pytest.mark.gpu

U, W = 2.0 ** -8, 2.0 ** -24


class Head:
    def __init__(self, T, H, V, masked=0.3, seed=0, std=None):
        g = torch.Generator().manual_seed(seed)
        self.T, self.H, self.V = T, H, V
        self.h = bf16_randn((T, H), seed + 1)
        self.e = bf16_randn((V, H), seed + 2, H ** -0.5 if std is None else std)
        t = torch.randint(0, V, (T,), generator=g, dtype=torch.int32)
        t[torch.rand(T, generator=g) < masked] = -1
        self.t = t.cuda()
        self.loss = torch.full((1,), 7.0, device="cuda")
        self.rows, self.lse = torch.full((T,), 7.0, device="cuda"), torch.full((T,), 7.0, device="cuda")
        self.dloss = torch.tensor([0.375], device="cuda")
        self.dh = torch.full((T, H), 7.0, dtype=torch.bfloat16, device="cuda")
        self.de = torch.full((V, H), 7.0, device="cuda")
        self.low = torch.full((V, H), 7.0, dtype=torch.bfloat16, device="cuda")

    def workspace(self, piece=0):
        return torch.empty(L.ls_head_loss_workspace(self.T, self.H, self.V, piece), dtype=torch.uint8, device="cuda")

    def fwd(self, ws=None, **kw):
        L.ls_head_loss_fwd(self.h, self.e, self.t, self.loss, self.rows, self.lse, self.workspace() if ws is None else ws, **kw)
        return self

    def bwd(self, de, piece=0, accumulate=False, dh=True, ws=None, dloss=True, **kw):
        L.ls_head_loss_bwd(self.h, self.e, self.t, self.lse, self.dloss if dloss else None, self.dh if dh else None, de,
                           accumulate, self.workspace(piece) if ws is None else ws, piece=piece, **kw)
        return self

    def reference(self, scale=0.375):
        h, e, t = self.h.double(), self.e.double(), self.t.long()
        z = h @ e.T
        lse = torch.logsumexp(z, 1)
        has = t >= 0
        n = max(int(has.sum()), 1)
        at = t.clamp(min=0)[:, None]
        rows = torch.where(has, lse - z.gather(1, at)[:, 0], 0.0)
        p = torch.exp(z - lse[:, None])
        c = scale / n
        dz = p.scatter_add(1, at, torch.full_like(at, -1.0, dtype=torch.float64)) * has[:, None] * c
        # how far the kernels may be
        ez = self.H * W * (h.abs() @ e.abs().T).amax(1)
        tol_lse = ez + 2.0 ** -17 + 2.0 ** -21 * lse.abs()
        edz = U * 1.01 * dz.abs() + c * p * (ez + tol_lse + 2.0 ** -17)[:, None] * has[:, None]
        dh, de = dz @ e, dz.T @ h
        tol_dh = edz @ e.abs() + self.V * W * (dz.abs() @ e.abs())
        tol_de = edz.T @ h.abs() + self.T * W * (dz.abs().T @ h.abs())
        return dict(lse=lse, rows=rows, loss=rows.sum() / n, dh=dh, de=de, tol_lse=tol_lse, tol_rows=tol_lse + ez,
                    tol_loss=(tol_lse + ez).amax() + 2.0 ** -23 * lse.abs().amax(), tol_dh=tol_dh * (1 + U) + U * dh.abs(),
                    tol_de=tol_de)


def within(name, got, ref, tol):
    err = (got.double() - ref).abs()
    assert bool((err <= tol).all()), (name, float((err / tol.clamp(min=1e-300)).max()))
    say(f"{name}: rel {float(err.norm() / ref.norm().clamp(min=1e-300)):.2e}, "
        f"worst share of the bound {float((err / tol.clamp(min=1e-300)).max()):.2f}")


def check_fwd(x, r):
    within("lse", x.lse, r["lse"], r["tol_lse"])
    within("row_loss", x.rows, r["rows"], r["tol_rows"])
    within("loss", x.loss[0], r["loss"], r["tol_loss"])


# one token; fewer rows than a tile and a vocabulary of any size; the rows around a workgroup's 64; whole tiles;
# more than one tile of every kind
SHAPES = [(1, 64, 100), (1, 2048, 3001), (3, 8, 50), (33, 24, 7), (5, 16, 1), (17, 40, 65), (7, 72, 1003), (64, 128, 129), (65, 128, 5), (130, 256, 512), (257, 128, 2049),
          (300, 320, 5000), (1025, 64, 20003)]


@pytest.mark.parametrize("T,H,V", SHAPES)
def test_matches_the_definition(T, H, V):
    need_gpu()
    say(T, H, V)
    x = Head(T, H, V, seed=T + V).fwd()
    r = x.reference()
    check_fwd(x, r)
    x.bwd(x.de)
    within("dh", x.dh, r["dh"], r["tol_dh"] + 1e-300)
    within("d_embed", x.de, r["de"], r["tol_de"] + 1e-300)
    x.bwd(x.low)
    within("d_embed bf16", x.low, r["de"], r["tol_de"] * (1 + U) + U * r["de"].abs() + 1e-300)


@pytest.mark.parametrize("T,H,V", [(2048, 256, 16390), (4099, 512, 8200)])
def test_large_tiles(T, H, V):
    """Shapes whose products run in 256 x 256 tiles, ragged on both sides."""
    need_gpu()
    x = Head(T, H, V, seed=5).fwd()
    r = x.reference()
    check_fwd(x, r)
    x.bwd(x.de).bwd(x.low, dh=False)
    within("dh", x.dh, r["dh"], r["tol_dh"])
    within("d_embed", x.de, r["de"], r["tol_de"])
    within("d_embed bf16", x.low, r["de"], r["tol_de"] * (1 + U) + U * r["de"].abs())


@pytest.mark.parametrize("piece", [0, 4096])
@pytest.mark.parametrize("T,H,V,masked", [(1500, 512, 9001, 0.8), (1500, 512, 9001, 0.97), (3000, 1024, 4500, 0.9),
                                          (509, 256, 33000, 0.5), (509, 256, 33000, 0.998), (700, 64, 20000, 1.0)])
def test_few_rows_with_a_target(T, H, V, masked, piece):
    """dh of few rows is split over the vocabulary by the device; the rows left out hold NaN."""
    need_gpu()
    x = Head(T, H, V, masked=masked, seed=11).fwd()
    r = x.reference()
    x.h[x.t < 0] = float("nan")
    x.bwd(x.de, piece=piece)
    within("dh", x.dh, r["dh"], r["tol_dh"] + 1e-300)
    within("d_embed", x.de, r["de"], r["tol_de"] + 1e-300)
    again = x.dh.clone()
    x.bwd(None, piece=piece)
    assert torch.equal(x.dh, again)


@pytest.mark.parametrize("piece", [1, 64, 200, 1024, 5000, 1 << 30])
def test_pieces(piece):
    need_gpu()
    x = Head(150, 192, 3003, seed=9).fwd()
    r = x.reference()
    x.bwd(x.de, piece=piece)
    within("dh", x.dh, r["dh"], r["tol_dh"])
    within("d_embed", x.de, r["de"], r["tol_de"])


@pytest.mark.parametrize("bm,bn", [(256, 256), (256, 192), (192, 256), (192, 192)])
def test_forced_tiles(bm, bn):
    """Whatever tile shape is forced on the products, with the workspace of the automatic choice."""
    need_gpu()
    x = Head(300, 256, 5003, seed=35)
    r = x.reference()
    ws = x.workspace()
    L.ls_gemm_tile_override(bm, bn)
    try:
        x.fwd(ws).bwd(x.de, ws=ws).bwd(x.low, dh=False, ws=ws)
        torch.cuda.synchronize()
    finally:
        L.ls_gemm_tile_override(0, 0)
    check_fwd(x, r)
    within("dh", x.dh, r["dh"], r["tol_dh"])
    within("d_embed", x.de, r["de"], r["tol_de"])
    within("d_embed bf16", x.low, r["de"], r["tol_de"] * (1 + U) + U * r["de"].abs())


def test_accumulate_and_wanted_outputs():
    need_gpu()
    x = Head(90, 128, 700, seed=11).fwd()
    r = x.reference()
    x.bwd(x.de, dh=False)
    assert (x.dh == 7).all()
    once = x.de.clone()
    x.bwd(x.de, accumulate=True)
    assert torch.equal(x.de, once + once)
    x.bwd(None)  # a frozen head
    within("dh", x.dh, r["dh"], r["tol_dh"])
    assert torch.equal(x.de, once + once)
    x.bwd(x.de, dloss=False)  # the loss's gradient is 1
    r1 = x.reference(scale=1.0)
    within("d_embed", x.de, r1["de"], r1["tol_de"])


def test_no_targets_at_all():
    need_gpu()
    x = Head(70, 64, 300, masked=1.1, seed=13).fwd()
    assert x.loss.item() == 0.0 and not x.rows.any()
    within("lse", x.lse, x.reference()["lse"], x.reference()["tol_lse"])
    x.bwd(x.de)
    assert not x.dh.any() and not x.de.any()


@pytest.mark.parametrize("T", [40, 200])
def test_targets_out_of_range(T):
    need_gpu()
    x = Head(T, 64, 300, masked=0.2, seed=15)
    x.t[3], x.t[17] = 300, -2
    x.fwd().bwd(x.de)
    bad = torch.zeros(T, dtype=torch.bool, device="cuda")
    bad[3] = bad[17] = True
    assert torch.equal(torch.isnan(x.rows), bad) and torch.isnan(x.loss).all()
    assert torch.equal(torch.isnan(x.dh).any(1), bad) and torch.isnan(x.dh[bad]).all()
    assert torch.isnan(x.de).all()
    y = Head(T, 64, 300, masked=0.2, seed=15)
    y.t[3] = y.t[17] = -1
    y.fwd().bwd(y.de)
    assert torch.equal(y.rows[~bad], x.rows[~bad]) and torch.equal(y.dh[~bad], x.dh[~bad])


def test_wide_range_of_logits():
    """Logits up to a hundred, some rows with one far above all others: no overflow, tiny losses stay right."""
    need_gpu()
    x = Head(96, 64, 1000, masked=0.1, seed=17, std=2.0).fwd()
    h, e = x.h.double(), x.e.double()
    z = h @ e.T
    ez = x.H * W * (h.abs() @ e.abs().T).amax(1)
    # exponents up to 2^8: 2^-16 relative on a term
    assert bool(((x.lse - torch.logsumexp(z, 1)).abs() <= ez + 2.0 ** -15 + 2.0 ** -21 * x.lse.abs()).all())
    assert torch.isfinite(x.loss).all()


def test_a_row_of_nan_stays_in_its_row():
    need_gpu()
    x = Head(100, 64, 500, masked=0.0, seed=19)
    y = Head(100, 64, 500, masked=0.0, seed=19)
    x.h[33] = float("nan")
    x.fwd().bwd(None)
    y.fwd().bwd(None)
    keep = torch.arange(100, device="cuda") != 33
    assert torch.equal(x.lse[keep], y.lse[keep]) and torch.equal(x.rows[keep], y.rows[keep])
    assert torch.equal(x.dh[keep], y.dh[keep])
    assert torch.isnan(x.lse[33]) and torch.isnan(x.loss).all() and torch.isnan(x.dh[33]).all()


@pytest.mark.parametrize("T,H,V", [(100, 64, 500), (700, 256, 9000)])
def test_rows_without_a_target_may_hold_anything(T, H, V):
    """Padding behind the last sequence: its h is NaN and reaches neither the loss nor a gradient."""
    need_gpu()
    x, y = Head(T, H, V, masked=0.6, seed=31), Head(T, H, V, masked=0.6, seed=31)
    none = x.t == -1
    assert bool(none.any()) and not bool(none.all())
    x.h[none] = float("nan")
    for a in (x, y):
        a.fwd().bwd(a.de).bwd(a.low, dh=False)
    assert torch.equal(x.loss, y.loss) and torch.equal(x.rows, y.rows)
    assert torch.equal(x.dh, y.dh) and not x.dh[none].any()
    assert torch.equal(x.de, y.de) and torch.equal(x.low, y.low)


@pytest.mark.parametrize("last", [True, False])
def test_a_single_target(last):
    need_gpu()
    x = Head(900, 256, 4000, masked=1.1, seed=33)
    x.t[899 if last else 0] = 77
    r = x.fwd().reference()
    check_fwd(x, r)
    x.bwd(x.de).bwd(x.low)
    within("dh", x.dh, r["dh"], r["tol_dh"] + 1e-300)
    within("d_embed", x.de, r["de"], r["tol_de"] + 1e-300)
    within("d_embed bf16", x.low, r["de"], r["tol_de"] * (1 + U) + U * r["de"].abs() + 1e-300)


def test_deterministic_and_no_stale_workspace():
    need_gpu()
    x = Head(333, 256, 4001, seed=21)
    ws = x.workspace()
    ws.fill_(255)  # NaN wherever floats are read
    x.fwd(ws)
    ws.fill_(255)
    x.bwd(x.de, ws=ws)
    first = [t.clone() for t in (x.loss, x.rows, x.lse, x.dh, x.de)]
    assert all(torch.isfinite(t).all() for t in first)
    ws.fill_(0)
    x.fwd(ws).bwd(x.de, ws=ws)
    assert all(torch.equal(a, b) for a, b in zip(first, (x.loss, x.rows, x.lse, x.dh, x.de)))


def test_nothing_written_outside_the_outputs():
    """Odd tokens and vocabulary: what lies behind each output stays."""
    need_gpu()
    T, H, V, pad = 131, 72, 1027, 4096
    x = Head(T, H, V, seed=23)
    out = {}
    for name, n, dt in (("rows", T, torch.float32), ("lse", T, torch.float32), ("dh", T * H, torch.bfloat16),
                        ("de", V * H, torch.float32), ("low", V * H, torch.bfloat16)):
        out[name] = torch.full((n + pad,), 5.0, dtype=dt, device="cuda")
    x.rows, x.lse = out["rows"][:T], out["lse"][:T]
    x.dh, x.de, x.low = out["dh"][:T * H].view(T, H), out["de"][:V * H].view(V, H), out["low"][:V * H].view(V, H)
    n = L.ls_head_loss_workspace(T, H, V)
    ws = torch.full((n + pad,), 9, dtype=torch.uint8, device="cuda")
    x.fwd(ws[:n]).bwd(x.de, ws=ws[:n]).bwd(x.low, ws=ws[:n]).bwd(x.de, piece=256, ws=ws[:n])
    for name, t in out.items():
        assert (t[-pad:] == 5).all(), name
    assert (ws[n:] == 9).all()
    r = x.reference()
    within("dh", x.dh, r["dh"], r["tol_dh"])


def test_head_weights_beyond_2_gib():
    """V x H x 2 = 2.4 GB: the forward takes the vocabulary in pieces too, and offsets pass 31 bits."""
    need_gpu()
    T, H, V = 24, 4096, 290_001
    g = torch.Generator(device="cuda")
    g.manual_seed(37)
    e = torch.empty(V, H, dtype=torch.bfloat16, device="cuda")
    for a in range(0, V, 50_000):
        e[a:a + 50_000] = torch.randn(min(50_000, V - a), H, generator=g, device="cuda") * H ** -0.5
    x = Head(T, H, 64, seed=37)
    x.V, x.e = V, e
    x.t = torch.tensor([0, V - 1, 261_990, 262_144, 131_072, -1] * 4, dtype=torch.int32, device="cuda")
    x.low = torch.full((V, H), 7.0, dtype=torch.bfloat16, device="cuda")
    x.fwd()
    h = x.h.double()
    z = torch.cat([h @ e[a:a + 20_000].double().T for a in range(0, V, 20_000)], 1)
    lse = torch.logsumexp(z, 1)
    has, at = x.t >= 0, x.t.long().clamp(min=0)
    rows = torch.where(has, lse - z.gather(1, at[:, None])[:, 0], 0.0)
    ez = H * W * (x.h.abs().double().sum(1) * float(e.abs().max()))
    tol = ez + 2.0 ** -17 + 2.0 ** -21 * lse.abs()
    within("lse", x.lse, lse, tol)
    within("row_loss", x.rows, rows, tol + ez)
    x.bwd(x.low)
    n = int(has.sum())
    dz = torch.exp(z - lse[:, None])
    dz[torch.arange(T, device="cuda"), at] -= 1.0
    dz *= has[:, None] * (0.375 / n)
    for v in (0, 1, 131_072, 261_990, 262_143, 262_144, V - 2, V - 1):
        ref = dz[:, v] @ h
        lim = (1.01 * U * dz[:, v].abs() + 2 * (tol * 0.375 / n) * torch.exp(z[:, v] - lse)) @ h.abs()
        within(f"d_embed[{v}]", x.low[v], ref, lim * (1 + U) + U * ref.abs() + T * W * (dz[:, v].abs() @ h.abs()))


def test_agrees_with_the_cross_entropy_of_kept_logits():
    """ls_gemm_nt and ls_cross_entropy round the logits to bf16: U/2 of the largest logit apart at most."""
    need_gpu()
    x = Head(256, 128, 1024, seed=25).fwd()
    z = torch.empty(256, 1024, dtype=torch.bfloat16, device="cuda")
    L.ls_gemm_nt(x.h, x.e, z)
    big = float(z.float().abs().max())
    loss, rows = torch.empty(1, device="cuda"), torch.empty(256, device="cuda")
    ws = torch.empty(L.ls_cross_entropy_workspace(256), dtype=torch.uint8, device="cuda")
    L.ls_cross_entropy(z, 256, x.t.clamp(min=0), x.t, loss, rows, ws)
    assert float((rows - x.rows).abs().max()) <= 2 * U * big
    assert abs(loss.item() - x.loss.item()) <= 2 * U * big


def test_capture_and_another_stream():
    need_gpu()
    x = Head(200, 128, 2000, seed=27)
    ws = x.workspace()

    def step():
        x.fwd(ws).bwd(x.de, ws=ws)

    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        step()
    torch.cuda.current_stream().wait_stream(s)
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        step()
    for i in range(3):
        x.h.copy_(bf16_randn(x.h.shape, 200 + i))
        x.t.copy_(torch.roll(x.t, 17 * i))
        step()
        torch.cuda.synchronize()
        want = [t.clone() for t in (x.loss, x.rows, x.lse, x.dh, x.de)]
        for t in (x.loss, x.rows, x.lse, x.dh, x.de):
            t.zero_()
        g.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(want, (x.loss, x.rows, x.lse, x.dh, x.de)))
    with torch.cuda.stream(s):
        x.fwd(ws, stream=s).bwd(x.de, ws=ws, stream=s)
    s.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(want, (x.loss, x.rows, x.lse, x.dh, x.de)))


def test_gradient_against_differences():
    need_gpu()
    x = Head(60, 64, 150, masked=0.2, seed=29).fwd()
    x.bwd(x.de)
    r = x.reference()
    g = torch.Generator().manual_seed(1)
    uh = torch.randn(60, 64, generator=g, dtype=torch.float64).cuda()
    ue = torch.randn(150, 64, generator=g, dtype=torch.float64).cuda()
    t, has = x.t.long(), x.t >= 0

    def loss(k):
        z = (x.h.double() + k * uh) @ (x.e.double() + k * ue).T
        rows = torch.logsumexp(z, 1) - z.gather(1, t.clamp(min=0)[:, None])[:, 0]
        return 0.375 * rows[has].sum() / has.sum()

    k = 1e-5
    change = (loss(k) - loss(-k)) / (2 * k)
    got = (x.dh.double() * uh).sum() + (x.de.double() * ue).sum()
    assert abs(got - change) <= (r["tol_dh"] * uh.abs()).sum() + (r["tol_de"] * ue.abs()).sum() + 1e-7
