"""Log probabilities, entropies, top alternatives and their gradients on the GPU against their definition in 64 bits.

Bounds count roundings: U = 2^-8 one rounding to bf16, W = 2^-24 one fp32 operation.  A scaled logit is an fp32 sum of H
products: off by ez = scale H W sum |h e|.  The log-sum-exp adds the exponent's rounding (2^-18 at |z| log2(e) < 2^6),
sums of V terms in blocks and a logarithm: 2^-17, and 2^-21 of its size for the factors scale log2(e) and ln 2.
The entropy's derivative by a logit is p (ln p + H), so that logits off by x move it by 2 x H at most; S and U are
good to 2^-17, and U / S is at most H: 2^-17 + H (2 ez + 2^-15).  A gradient's entry g (onehot - p) - e p (ln p + H) is
off by p (|g| + |e| (|ln p + H| + 1)) for ln p's error and |e| p for the entropy's, then rounded to bf16."""
from __future__ import annotations

import pytest
import torch

from gpu_util import bf16_randn, need_gpu, say
from paper_2510_02483_amd import lib as L

pytestmark = pytest.mark.gpu

U, W = 2.0 ** -8, 2.0 ** -24
F32, I32, BF16 = torch.float32, torch.int32, torch.bfloat16


def full(*shape, dtype=F32):
    return torch.full(shape, 7, dtype=dtype, device="cuda")


class Head:
    def __init__(self, T, H, V, top=0, scale=1.0, masked=0.3, seed=0, std=None, integers=False):
        g = torch.Generator().manual_seed(seed)
        self.T, self.H, self.V, self.top, self.scale = T, H, V, top, scale
        if integers:  # every sum of products is exact in 32 bits, equal logits are many
            self.h = torch.randint(-2, 3, (T, H), generator=g).to(BF16).cuda()
            self.e = torch.randint(-2, 3, (V, H), generator=g).to(BF16).cuda()
        else:
            self.h = bf16_randn((T, H), seed + 1)
            self.e = bf16_randn((V, H), seed + 2, H ** -0.5 if std is None else std)
        t = torch.randint(0, V, (T,), generator=g, dtype=I32)
        t[torch.rand(T, generator=g) < masked] = -1
        self.t = t.cuda()
        self.dlp, self.den = (torch.randn(T, generator=g) * 0.3).cuda(), (torch.randn(T, generator=g) * 0.1).cuda()
        self.logprob, self.entropy, self.lse = full(T), full(T), full(T)
        self.ids, self.vals = full(T, top, dtype=I32), full(T, top)
        self.dh, self.de, self.low = full(T, H, dtype=BF16), full(V, H), full(V, H, dtype=BF16)

    def workspace(self, piece=0):
        return torch.empty(L.ls_token_logprob_workspace(self.T, self.H, self.V, self.top, piece), dtype=torch.uint8,
                           device="cuda")

    def fwd(self, ws=None, **kw):
        if self.top:
            kw.update(top_ids=self.ids, top_logprob=self.vals)
        L.ls_token_logprob_fwd(self.h, self.e, self.t, self.logprob, self.entropy, self.lse,
                               self.workspace() if ws is None else ws, scale=self.scale, **kw)
        return self

    def bwd(self, de, piece=0, accumulate=False, dh=True, ws=None, dlp=True, den=True, **kw):
        L.ls_token_logprob_bwd(self.h, self.e, self.t, self.entropy, self.lse, self.dlp if dlp else None,
                               self.den if den else None, self.dh if dh else None, de, accumulate,
                               self.workspace(piece) if ws is None else ws, scale=self.scale, piece=piece, **kw)
        return self

    def reference(self, dlp=True, den=True):
        h, e, t = self.h.double(), self.e.double(), self.t.long()
        has, at = t >= 0, t.clamp(min=0)[:, None]
        z = h @ e.T * self.scale
        self.z = z
        lse = torch.logsumexp(z, 1)
        ln = z - lse[:, None]
        p = ln.exp()
        ent = -(p * ln).sum(1)
        ez = self.scale * self.H * W * (h.abs() @ e.abs().T).amax(1)
        tol_lse = ez + 2.0 ** -17 + 2.0 ** -21 * lse.abs()
        tol_ent = 2.0 ** -17 + ent * (2 * ez + 2.0 ** -15)
        r = dict(lse=lse, logprob=torch.where(has, ln.gather(1, at)[:, 0], 0.0), entropy=torch.where(has, ent, 0.0),
                 tol_lse=tol_lse, tol_logprob=tol_lse + ez, tol_entropy=tol_ent)
        g = self.dlp.double()[:, None] * has[:, None] * dlp
        b = self.den.double()[:, None] * has[:, None] * den
        slope = (ln + ent[:, None]).abs()
        one = torch.zeros_like(p).scatter_(1, at, 1.0)
        dz = g * (one - p) - b * p * (ln + ent[:, None])
        off = p * (g.abs() + b.abs() * (slope + 1))
        edz = 1.01 * U * dz.abs() + off * (ez + tol_lse + 2.0 ** -17)[:, None] + p * b.abs() * tol_ent[:, None] + \
            2.0 ** -22 * (off + one * g.abs())
        s = self.scale
        tol_dh = edz @ e.abs() + self.V * W * (dz.abs() @ e.abs())
        tol_de = edz.T @ h.abs() + self.T * W * (dz.abs().T @ h.abs())
        r.update(dh=s * dz @ e, de=s * dz.T @ h, tol_de=s * tol_de + 1e-37)
        r["tol_dh"] = s * tol_dh * (1 + U) + U * r["dh"].abs() + 1e-37
        return r


def within(name, got, ref, tol):
    err = (got.double() - ref).abs()
    assert bool((err <= tol).all()), (name, float((err / tol.clamp(min=1e-300)).max()))
    say(f"{name}: rel {float(err.norm() / ref.norm().clamp(min=1e-300)):.2e}, "
        f"worst share of the bound {float((err / tol.clamp(min=1e-300)).max()):.2f}")


def check_fwd(x, r):
    for name in ("lse", "logprob", "entropy"):
        within(name, getattr(x, name), r[name], r["tol_" + name])
    if x.top:
        check_top(x, r)


def check_top(x, r):
    """Values of the ids that are named, no id twice, in order, and none that was left out above the last by more
    than the roundings."""
    k = min(x.top, x.V)
    ids, vals = x.ids[:, :k].long(), x.vals[:, :k]
    assert (x.ids[:, k:] == -1).all() and torch.isneginf(x.vals[:, k:]).all()
    assert ((ids >= 0) & (ids < x.V)).all()
    assert (torch.sort(ids, 1).values.diff(dim=1) > 0).all() and (vals.diff(dim=1) <= 0).all()
    ln = x.z - r["lse"][:, None]
    tol = r["tol_logprob"][:, None]
    within("top values", vals, ln.gather(1, ids), tol.expand_as(ids))
    rest = ln.scatter(1, ids, float("-inf"))
    assert (rest.amax(1, keepdim=True) <= ln.gather(1, ids).amin(1, keepdim=True) + 2 * tol).all()


def check_bwd(x, r, low=False):
    within("dh", x.dh, r["dh"], r["tol_dh"])
    within("d_embed", x.de, r["de"], r["tol_de"])
    if low:
        within("d_embed bf16", x.low, r["de"], r["tol_de"] * (1 + U) + U * r["de"].abs())


# one token; fewer rows than a tile and a vocabulary of any size; the rows around a workgroup's; whole tiles; more
# than one tile of every kind; more rows than one workgroup each serves
SHAPES = [(1, 64, 100, 8), (1, 2048, 3001, 64), (3, 8, 50, 1), (33, 24, 7, 9), (5, 16, 1, 2), (17, 40, 65, 64), (7, 72, 1003, 17),
          (64, 128, 129, 3), (65, 128, 16, 4), (130, 256, 512, 5), (257, 128, 2049, 64), (300, 320, 5000, 2),
          (512, 64, 1500, 16), (513, 64, 1500, 16), (1022, 64, 9000, 8), (1024, 72, 900, 17), (1025, 64, 20003, 6), (1040, 128, 33, 33)]


@pytest.mark.parametrize("T,H,V,top", SHAPES)
def test_matches_the_definition(T, H, V, top):
    need_gpu()
    say(T, H, V, top)
    x = Head(T, H, V, top, scale=[1.0, 1.25, 0.5][T % 3], seed=T + V, masked=0.3 if T > 1 else 0.0).fwd()
    r = x.reference()
    check_fwd(x, r)
    x.bwd(x.de).bwd(x.low)
    check_bwd(x, r, low=True)


@pytest.mark.parametrize("T,H,V,top", [(2048, 256, 16390, 8), (4099, 512, 8200, 0), (1, 512, 131072, 8)])
def test_large_tiles(T, H, V, top):
    need_gpu()
    x = Head(T, H, V, top, scale=1.25, seed=5, masked=0.0).fwd()
    r = x.reference()
    check_fwd(x, r)
    x.bwd(x.de).bwd(x.low, dh=False)
    check_bwd(x, r, low=True)


@pytest.mark.parametrize("T,V,top", [(1, 40, 12), (70, 300, 64), (70, 2000, 8), (1100, 700, 8), (1100, 17, 20), (1030, 5000, 64)])
def test_equal_logits_go_to_the_lower_token(T, V, top):
    need_gpu()
    x = Head(T, 16, V, top, seed=T, integers=True, scale=0.5).fwd()
    order = torch.sort(x.h.double() @ x.e.double().T, dim=1, descending=True, stable=True).indices[:, :top].int()
    k = min(top, V)
    assert torch.equal(x.ids[:, :k], order)
    assert (x.ids[:, k:] == -1).all() and torch.isneginf(x.vals[:, k:]).all()
    r = x.reference()
    check_fwd(x, r)


def test_all_logits_equal():
    need_gpu()
    for T in (5, 1030):
        x = Head(T, 64, 1000, 20, seed=1, masked=0.0)
        x.h.zero_()
        x.fwd()
        assert (x.ids == torch.arange(20, device="cuda", dtype=I32)).all()
        ln = torch.log(torch.tensor(1000.0, dtype=torch.float64)).item()
        assert float((x.entropy.double() - ln).abs().max()) <= 2.0 ** -17 + ln * 2.0 ** -15
        assert float((x.vals.double() + ln).abs().max()) <= 2.0 ** -17 + ln * 2.0 ** -21


@pytest.mark.parametrize("T", [2, 601, 1030])
@pytest.mark.parametrize("top", [1, 16, 17, 64])
@pytest.mark.parametrize("low", [None, 0, 5, 15])
def test_logits_in_any_arrangement(T, top, low):
    """Rising, falling and constant along the vocabulary, and far lower in every 16th stretch of 512 tokens."""
    need_gpu()
    V = 20_003
    x = Head(T, 16, V, top, seed=3, masked=0.0)
    x.h.zero_()
    x.h[0, 0] = 1.0
    x.h[1, 0] = -1.0
    x.h[T - 1, 1] = 1.0
    v = torch.arange(V, device="cuda")
    x.e.zero_()
    x.e[:, 0] = (v // 100).to(BF16)  # whole numbers up to 200: exact
    x.e[:, 1] = (v % 7).to(BF16)
    if low is not None:
        x.e[(v // 512) % 16 == low] -= 250.0 if T > 2 else 256.0
    x.fwd()
    z = x.h.double() @ x.e.double().T
    assert torch.equal(x.ids, torch.sort(z, dim=1, descending=True, stable=True).indices[:, :top].int())


@pytest.mark.parametrize("piece", [0, 4096])
@pytest.mark.parametrize("T,H,V,masked", [(1500, 512, 9001, 0.8), (1500, 512, 9001, 0.97), (509, 256, 33000, 0.998)])
def test_few_rows_with_a_target(T, H, V, masked, piece):
    """The rows left out of the gradients hold NaN, and so do their gradients."""
    need_gpu()
    x = Head(T, H, V, masked=masked, seed=11).fwd()
    r = x.reference()
    for t in (x.h, x.dlp, x.den, x.lse, x.entropy):
        t[x.t < 0] = float("nan")
    x.bwd(x.de, piece=piece)
    check_bwd(x, r)
    again = x.dh.clone()
    x.bwd(None, piece=piece)
    assert torch.equal(x.dh, again)


@pytest.mark.parametrize("piece", [1, 64, 200, 1024, 5000, 1 << 30])
def test_pieces(piece):
    need_gpu()
    x = Head(150, 192, 3003, seed=9).fwd()
    r = x.reference()
    x.bwd(x.de, piece=piece)
    check_bwd(x, r)


@pytest.mark.parametrize("bm,bn", [(256, 256), (256, 192), (192, 256), (192, 192)])
def test_forced_tiles(bm, bn):
    """Whatever tile shape is forced on the products, with the workspace of the automatic choice."""
    need_gpu()
    x = Head(300, 256, 5003, 8, seed=35)
    r = x.reference()
    ws = x.workspace()
    L.ls_gemm_tile_override(bm, bn)
    try:
        x.fwd(ws).bwd(x.de, ws=ws).bwd(x.low, dh=False, ws=ws)
        torch.cuda.synchronize()
    finally:
        L.ls_gemm_tile_override(0, 0)
    check_fwd(x, r)
    check_bwd(x, r, low=True)


@pytest.mark.parametrize("dlp,den", [(True, False), (False, True)])
def test_one_gradient_alone(dlp, den):
    need_gpu()
    x = Head(90, 128, 700, seed=11).fwd()
    x.bwd(x.de, dlp=dlp, den=den)
    check_bwd(x, x.reference(dlp, den))
    one = x.dh.clone(), x.de.clone()
    (x.den if dlp else x.dlp).zero_()
    x.bwd(x.de)
    assert torch.equal(one[0], x.dh) and torch.equal(one[1], x.de)


def test_accumulate_and_wanted_outputs():
    need_gpu()
    x = Head(90, 128, 700, seed=11).fwd()
    r = x.reference()
    x.bwd(x.de, dh=False)
    assert (x.dh == 7).all()
    once = x.de.clone()
    x.bwd(x.de, accumulate=True)
    assert torch.equal(x.de, once + once)
    x.bwd(None)
    within("dh", x.dh, r["dh"], r["tol_dh"])
    assert torch.equal(x.de, once + once)


def test_gradients_of_zero_and_no_targets():
    need_gpu()
    x = Head(70, 64, 300, 4, masked=1.1, seed=13).fwd()
    assert not x.logprob.any() and not x.entropy.any()
    check_fwd(x, x.reference())  # lse and alternatives of every row all the same
    x.bwd(x.de)
    assert not x.dh.any() and not x.de.any()
    x = Head(70, 64, 300, seed=13).fwd()
    x.dlp.zero_()
    x.den.zero_()
    x.bwd(x.de)
    assert not x.dh.any() and not x.de.any()


@pytest.mark.parametrize("g", [1e-30, 1e30])
def test_gradients_of_any_size(g):
    """A common factor of the rows' gradients leaves, and rows far below the largest keep their bits."""
    need_gpu()
    x = Head(60, 64, 300, masked=0.0, seed=13)
    x.dlp *= g
    x.den *= g
    x.dlp[:20] *= 2.0 ** -20
    x.den[:20] *= 2.0 ** -20
    x.fwd().bwd(x.de)
    check_bwd(x, x.reference())


@pytest.mark.parametrize("T", [40, 200])
def test_targets_out_of_range(T):
    need_gpu()
    x = Head(T, 64, 300, masked=0.2, seed=15)
    x.t[3], x.t[17] = 300, -2
    x.fwd().bwd(x.de)
    bad = torch.zeros(T, dtype=torch.bool, device="cuda")
    bad[3] = bad[17] = True
    assert torch.equal(torch.isnan(x.logprob), bad) and torch.equal(torch.isnan(x.entropy), bad)
    assert torch.isfinite(x.lse).all()
    assert torch.equal(torch.isnan(x.dh).any(1), bad) and torch.isnan(x.dh[bad]).all()
    assert torch.isnan(x.de).all()


@pytest.mark.parametrize("bad", [float("nan"), float("inf")])
@pytest.mark.parametrize("which", ["dlp", "den"])
def test_gradients_that_are_no_numbers(bad, which):
    need_gpu()
    x, y = Head(70, 64, 300, masked=0.0, seed=15).fwd(), Head(70, 64, 300, masked=0.0, seed=15).fwd()
    getattr(x, which)[33] = bad
    getattr(y, which)[33] = 0.0
    x.bwd(x.de)
    y.bwd(y.de)
    keep = torch.arange(70, device="cuda") != 33
    assert torch.isnan(x.dh[33]).all() and torch.isnan(x.de).all() and torch.equal(x.dh[keep], y.dh[keep])


def test_wide_range_of_logits():
    """Logits up to hundreds, some rows with one far above all others: no overflow, entropies from 0 up."""
    need_gpu()
    x = Head(96, 64, 1000, 5, masked=0.0, seed=17, std=6.0)
    r = x.fwd().reference()
    big = x.z.abs().amax(1)
    assert 2.0 ** 7 < float(big.max()) * 1.443 < 2.0 ** 10
    wide = 2.0 ** -14  # exponents up to 2^10: 2^-14 on a term
    within("lse", x.lse, r["lse"], r["tol_lse"] + wide)
    within("logprob", x.logprob, r["logprob"], r["tol_logprob"] + wide + 2.0 ** -21 * big)
    within("entropy", x.entropy, r["entropy"], r["tol_entropy"] + r["entropy"] * 2.0 ** -12 + 2.0 ** -20)
    x.bwd(x.de)
    assert torch.isfinite(x.dh).all() and torch.isfinite(x.de).all()


def test_infinite_logits():
    """Tokens whose logit is -inf have no probability and add no entropy; among the alternatives they come last."""
    need_gpu()
    x = Head(50, 8, 300, 37, masked=0.0, seed=18)
    x.h[:, 0] = 1.0
    x.e[100:, 0] = float("-inf")
    x.t %= 100
    x.fwd()
    y = Head(50, 8, 100, x.top, masked=0.0, seed=18)
    y.h.copy_(x.h)
    y.e.copy_(x.e[:100])
    y.t.copy_(x.t)
    r = y.reference()
    for name in ("lse", "logprob", "entropy"):
        within(name, getattr(x, name), r[name], r["tol_" + name])
    y.ids, y.vals = x.ids, x.vals
    check_top(y, r)
    p = Head(50, 8, 300, 64, masked=0.0, seed=18)
    p.h.copy_(x.h)
    p.e.copy_(x.e)
    p.e[40:, 0] = float("-inf")
    p.t.copy_(x.t % 40)
    p.fwd()
    assert (p.ids[:, :40] < 40).all() and torch.isneginf(p.vals[:, 40:]).all()
    assert torch.equal(p.ids[:, 40:], torch.arange(40, 64, dtype=I32, device="cuda").expand(50, 24))


@pytest.mark.parametrize("T", [100, 1100])
def test_a_row_of_nan_stays_in_its_row(T):
    need_gpu()
    x, y = (Head(T, 64, 500, 4, masked=0.0, seed=19) for _ in range(2))
    x.h[33] = float("nan")
    x.fwd().bwd(None)
    y.fwd().bwd(None)
    keep = torch.arange(T, device="cuda") != 33
    for a, b in ((x.lse, y.lse), (x.logprob, y.logprob), (x.entropy, y.entropy), (x.dh, y.dh), (x.ids, y.ids), (x.vals, y.vals)):
        assert torch.equal(a[keep], b[keep])
    assert torch.isnan(x.lse[33]) and torch.isnan(x.logprob[33]) and torch.isnan(x.entropy[33]) and torch.isnan(x.dh[33]).all()
    assert (x.ids[33] == -1).all()


@pytest.mark.parametrize("T", [20, 1100])
def test_nan_logits_are_no_alternatives(T):
    need_gpu()
    x, y = (Head(T, 64, 500, 9, masked=0.0, seed=19) for _ in range(2))
    x.e[::7] = float("nan")
    y.e[::7] = 0.0
    y.e[::7, 0] = float("-inf")
    y.h[:, 0] = x.h[:, 0] = x.h[:, 0].abs() + 1.0
    x.fwd()
    y.fwd()
    assert torch.isnan(x.lse).all() and torch.equal(x.ids, y.ids)


def test_deterministic_and_no_stale_workspace():
    need_gpu()
    x = Head(333, 256, 4001, 8, seed=21)
    outs = (x.logprob, x.entropy, x.lse, x.ids, x.vals, x.dh, x.de)
    ws = x.workspace()
    ws.fill_(255)
    x.fwd(ws)
    ws.fill_(255)
    x.bwd(x.de, ws=ws)
    first = [t.clone() for t in outs]
    assert all(torch.isfinite(t.float()).all() for t in first)
    ws.fill_(0)
    x.fwd(ws).bwd(x.de, ws=ws)
    assert all(torch.equal(a, b) for a, b in zip(first, outs))


@pytest.mark.parametrize("T,V", [(131, 1027), (1027, 131), (1, 257)])
def test_nothing_written_outside_the_outputs(T, V):
    need_gpu()
    H, k, pad = 72, 5, 4096
    x = Head(T, H, V, k, seed=23, masked=0.0)
    out = {}
    for name, n, dt in (("logprob", T, F32), ("entropy", T, F32), ("lse", T, F32), ("ids", T * k, I32), ("vals", T * k, F32),
                        ("dh", T * H, BF16), ("de", V * H, F32), ("low", V * H, BF16)):
        out[name] = torch.full((n + pad,), 5, dtype=dt, device="cuda")
        setattr(x, name, out[name][:n].view(getattr(x, name).shape))
    n = L.ls_token_logprob_workspace(T, H, V, k)
    ws = torch.full((n + pad,), 9, dtype=torch.uint8, device="cuda")
    x.fwd(ws[:n]).bwd(x.de, ws=ws[:n]).bwd(x.low, ws=ws[:n]).bwd(x.de, piece=256, ws=ws[:n])
    for name, t in out.items():
        assert (t[-pad:] == 5).all(), name
    assert (ws[n:] == 9).all()
    r = x.reference()
    check_fwd(x, r)
    check_bwd(x, r, low=True)


def test_head_weights_beyond_2_gib():
    """V x H x 2 = 2.4 GB: the vocabulary in pieces, and offsets pass 31 bits."""
    need_gpu()
    T, H, V = 24, 4096, 290_001
    g = torch.Generator(device="cuda")
    g.manual_seed(37)
    e = torch.empty(V, H, dtype=BF16, device="cuda")
    for a in range(0, V, 50_000):
        e[a:a + 50_000] = torch.randn(min(50_000, V - a), H, generator=g, device="cuda") * H ** -0.5
    x = Head(T, H, 64, 6, seed=37)
    x.V, x.e = V, e
    x.t = torch.tensor([0, V - 1, 261_990, 262_144, 131_072, -1] * 4, dtype=I32, device="cuda")
    e[V - 1] = x.h[3] / 8.0  # far above all others in one row
    x.low = full(V, H, dtype=BF16)
    x.fwd()
    h = x.h.double()
    z = torch.cat([h @ e[a:a + 20_000].double().T for a in range(0, V, 20_000)], 1)
    lse = torch.logsumexp(z, 1)
    ln = z - lse[:, None]
    ent = -(ln.exp() * ln).sum(1)
    has, at = x.t >= 0, x.t.long().clamp(min=0)
    ez = H * W * (x.h.abs().double().sum(1) * float(e.abs().max()))
    tol = ez + 2.0 ** -17 + 2.0 ** -21 * lse.abs()
    big = z.abs().amax(1)
    wide = 2.0 ** -14 * (big > 40)
    within("lse", x.lse, lse, tol + wide)
    within("logprob", x.logprob, torch.where(has, ln.gather(1, at[:, None])[:, 0], 0.0), tol + ez + wide)
    within("entropy", x.entropy, torch.where(has, ent, 0.0), 2.0 ** -17 + ent * (2 * ez + 2.0 ** -15) + wide)
    assert x.ids[3, 0] == V - 1
    top = torch.sort(z, 1, descending=True).values[:, :6] - lse[:, None]
    within("top", x.vals, top, (tol + 2 * ez + wide)[:, None].expand_as(top))
    x.bwd(x.low)
    one = torch.zeros_like(z).scatter_(1, at[:, None], 1.0)
    gl, ge = x.dlp.double()[:, None] * has[:, None], x.den.double()[:, None] * has[:, None]
    dz = gl * (one - ln.exp()) - ge * ln.exp() * (ln + ent[:, None])
    for v in (0, 1, 131_072, 261_990, 262_143, 262_144, V - 2, V - 1):
        p = ln[:, v].exp()
        off = p * (gl[:, 0].abs() + ge[:, 0].abs() * ((ln[:, v] + ent).abs() + 2))
        lim = (1.01 * U * dz[:, v].abs() + off * (2 * tol + wide + ent * (2 * ez + 2.0 ** -15)) +
               2.0 ** -22 * one[:, v] * gl[:, 0].abs()) @ h.abs()
        ref = dz[:, v] @ h
        within(f"d_embed[{v}]", x.low[v], ref, lim * (1 + U) + U * ref.abs() + T * W * (dz[:, v].abs() @ h.abs()))


def test_agrees_with_the_head_loss():
    """The mean of -logprob is the head's loss, and gradients of -1 / N give its gradients."""
    need_gpu()
    x = Head(256, 128, 1024, seed=25).fwd()
    r = x.reference()
    loss, rows, lse = full(1), full(256), full(256)
    ws = torch.empty(L.ls_head_loss_workspace(256, 128, 1024), dtype=torch.uint8, device="cuda")
    L.ls_head_loss_fwd(x.h, x.e, x.t, loss, rows, lse, ws)
    assert bool(((rows + x.logprob).abs() <= 2 * r["tol_logprob"]).all())
    n = int((x.t >= 0).sum())
    x.dlp.fill_(-1.0 / n)
    x.bwd(x.de, den=False)
    dh, de = torch.empty_like(x.dh), torch.empty_like(x.de)
    L.ls_head_loss_bwd(x.h, x.e, x.t, lse, None, dh, de, False, ws)
    r = x.reference(den=False)
    assert bool(((dh.double() - x.dh.double()).abs() <= 2 * r["tol_dh"]).all())
    assert bool(((de.double() - x.de.double()).abs() <= 2 * r["tol_de"]).all())


def test_capture_and_two_streams():
    """A captured step replayed between eager ones on other data, two streams with a workspace each at once."""
    need_gpu()
    x = Head(200, 128, 2000, 8, seed=27)
    outs = (x.logprob, x.entropy, x.lse, x.ids, x.vals, x.dh, x.de)
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
        x.dlp.copy_(torch.roll(x.dlp, 3))
        step()
        torch.cuda.synchronize()
        want = [t.clone() for t in outs]
        for t in outs:
            t.zero_()
        g.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(want, outs))
    y = Head(200, 128, 2000, 8, seed=28)
    ws2 = y.workspace()
    torch.cuda.synchronize()
    y.fwd(ws2).bwd(y.de, ws=ws2)
    ref = [t.clone() for t in (y.logprob, y.ids, y.dh, y.de)]
    torch.cuda.synchronize()
    with torch.cuda.stream(s):
        x.fwd(ws, stream=s).bwd(x.de, ws=ws, stream=s)
    y.fwd(ws2).bwd(y.de, ws=ws2)
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(want, outs))
    assert all(torch.equal(a, b) for a, b in zip(ref, (y.logprob, y.ids, y.dh, y.de)))


def test_gradient_against_differences():
    need_gpu()
    x = Head(60, 64, 150, scale=1.25, masked=0.2, seed=29).fwd()
    x.bwd(x.de)
    r = x.reference()
    g = torch.Generator().manual_seed(1)
    uh = torch.randn(60, 64, generator=g, dtype=torch.float64).cuda()
    ue = torch.randn(150, 64, generator=g, dtype=torch.float64).cuda()
    t, has = x.t.long(), x.t >= 0

    def loss(k):
        ln = torch.log_softmax((x.h.double() + k * uh) @ (x.e.double() + k * ue).T * 1.25, 1)
        row = x.dlp.double() * ln.gather(1, t.clamp(min=0)[:, None])[:, 0] - x.den.double() * (ln.exp() * ln).sum(1)
        return row[has].sum()

    k = 1e-5
    change = (loss(k) - loss(-k)) / (2 * k)
    got = (x.dh.double() * uh).sum() + (x.de.double() * ue).sum()
    assert abs(got - change) <= (r["tol_dh"] * uh.abs()).sum() + (r["tol_de"] * ue.abs()).sum() + 1e-7
