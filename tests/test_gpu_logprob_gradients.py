"""Gradients of log probabilities and entropies against differences of the loss, and over a wide range of logits."""
from __future__ import annotations

import pytest
import torch

from gpu_util import need_gpu, say
from test_gpu_logprob import U, Head, within

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dlp,den", [(True, False), (False, True), (True, True)])
@pytest.mark.parametrize("which", ["h", "e"])
def test_differences_in_one_operand(which, dlp, den):
    """Random directions in h alone or in the head's weights alone, for either gradient.

    Every entry of dz is rounded once, to U of itself, and so is one of dh: with independent roundings, what reaches the
    product with a direction has a standard deviation of at most U |dz * w| and U |dh * u|, w = scale u e^T (or h u^T) what
    the direction adds to the logits.  Five of them are allowed, and 4% for the roundings in fp32."""
    need_gpu()
    x = Head(60, 64, 150, scale=1.25, masked=0.2, seed=29).fwd()
    x.bwd(x.de, dlp=dlp, den=den)
    h, e, t, has = x.h.double(), x.e.double(), x.t.long(), (x.t >= 0).double()
    a = x.dlp.double() * has * dlp
    b = x.den.double() * has * den

    def loss(h, e):
        ln = torch.log_softmax(h @ e.T * 1.25, 1)
        return (a * ln.gather(1, t.clamp(min=0)[:, None])[:, 0] - b * (ln.exp() * ln).sum(1)).sum()

    z = (h @ e.T * 1.25).requires_grad_()
    ln = torch.log_softmax(z, 1)
    (a * ln.gather(1, t.clamp(min=0)[:, None])[:, 0] - b * (ln.exp() * ln).sum(1)).sum().backward()
    got = (x.dh if which == "h" else x.de).double()
    g = torch.Generator().manual_seed(1)
    changes, limits = [], []
    for _ in range(6):
        u = torch.randn(got.shape, generator=g, dtype=torch.float64).cuda()
        k = 1e-5
        if which == "h":
            change, w = (loss(h + k * u, e) - loss(h - k * u, e)) / (2 * k), 1.25 * u @ e.T
        else:
            change, w = (loss(h, e + k * u) - loss(h, e - k * u)) / (2 * k), 1.25 * h @ u.T
        lim = 5.2 * U * ((z.grad * w).norm() + ((got * u).norm() if which == "h" else 0.0)) + 1e-8
        off = abs((got * u).sum() - change)
        say(f"change {float(change):.4f} off {float(off):.2e} limit {float(lim):.2e}")
        assert off <= lim
        changes.append(abs(float(change)))
        limits.append(float(lim))
    # (so that a gradient of nothing, or of a part, cannot pass)
    assert max(limits) < 0.1 * max(changes)


@pytest.mark.parametrize("dlp,den", [(True, False), (False, True), (True, True)])
def test_gradients_of_a_wide_range_of_logits(dlp, den):
    """Logits up to hundreds, rows whose entropy is next to 0: the terms of dz cancel there.

    ln p comes from a logit and a log-sum-exp of up to 2^10 in base 2: the latter's two roundings and two constants, 3 x
    2^-14, so 2^-12 beside what Head.reference counts; the entropy is good to 2^-12 of itself and 2^-20 here.  Probabilities
    below 2^-126, the smallest that exp2 gives, are 0, and so are entries of dz / c below it, c the largest gradient: d_embed
    of token 254 is 3.2e-36, of which a row whose p is 3.3e-39 has 1.5e-37."""
    need_gpu()
    x = Head(96, 64, 1000, masked=0.1, seed=17, std=6.0).fwd()
    x.bwd(x.de, dlp=dlp, den=den)
    r = x.reference(dlp, den)
    assert 2.0 ** 7 < float(x.z.abs().max()) * 1.443 < 2.0 ** 10
    assert float((r["entropy"][x.t >= 0] < 1e-3).double().mean()) > 0.2
    h, e, has = x.h.double(), x.e.double(), (x.t >= 0).double()[:, None]
    ln = x.z - r["lse"][:, None]
    p = ln.exp()
    ent = -(p * ln).sum(1, keepdim=True)
    g, b = x.dlp.double().abs()[:, None] * has * dlp, x.den.double().abs()[:, None] * has * den
    slope = (ln + ent).abs()
    more = p * (g + b * (slope + 1)) * 2.0 ** -12 + p * b * (ent * 2.0 ** -12 + 2.0 ** -20)
    more += p.clamp(max=2.0 ** -126) * (g + b * slope) + 2.0 ** -126 * torch.maximum(g.max(), b.max()) * has
    within("dh", x.dh, r["dh"], r["tol_dh"] + more @ e.abs() * (1 + U))
    within("d_embed", x.de, r["de"], r["tol_de"] + more.T @ h.abs())
