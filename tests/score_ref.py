"""Capped and windowed attention, and q/k norm with rotation, over packed sequences in 64 bits, and how far the kernels
may be from them.  Bounds count roundings (U, W as in packed_ref)."""
from __future__ import annotations

import numpy as np

import packed_ref as R

U, W = R.U, R.W


def attention(qkv, lens, first, nq, nkv, d, dout=None, scale=0.0, cap=0.0, window=0, rest=False):
    """packed_ref.attention with scores cap tanh(scale q.k / cap) over a window.

    Beside the errors counted there: a capped score is c2 - 2 c2 r with r good to 1.9 x 2^-23, so it is off by cap x
    2^-21, and p relatively by twice that (its own and the log-sum-exp's); the slope 4 r (1 - r) is off by 2^-20.
    rest: D comes from o and the rest of its rounding, which is o to 2^-17 but for the rounding of p."""
    total = qkv.shape[0]
    o, lse, grad = np.zeros((total, nq * d)), np.zeros((nq, total)), np.zeros_like(qkv)
    tol = {"o": np.zeros_like(o), "lse": np.zeros_like(lse), "dqkv": np.zeros_like(qkv)}
    at = R.bounds_of(lens, first)
    sc = scale or 1.0 / np.sqrt(d)
    off = cap * 2.0 ** -21
    for a, b in zip(at, at[1:]):
        n = int(b - a)
        if n == 0:
            continue
        far = np.arange(n)[:, None] - np.arange(n)[None, :]
        seen = (far >= 0) & (far < (window or n))
        for h in range(nq):
            g = h // (nq // nkv)
            hq, hk, hv = (slice(x * d, (x + 1) * d) for x in (h, nq + g, nq + nkv + g))
            q, k, v = qkv[a:b, hq], qkv[a:b, hk], qkv[a:b, hv]
            raw = q @ k.T * sc
            slope = np.ones_like(raw)
            if cap:
                t = np.tanh(raw / cap)
                slope, raw = 1 - t * t, cap * t
            s = np.where(seen, raw, -np.inf)
            m = s.max(1, keepdims=True)
            e = np.exp(s - m)
            l = e.sum(1, keepdims=True)
            p = e / l
            # the exponent's fp32 error: that of a score of d products, and of its own size
            big = np.abs(np.where(seen, s, 0.0)).max()
            slack = 2.0 ** -18 + 2 * off + 2.0 ** -22 * big
            o[a:b, hq] = p @ v
            lse[h, a:b] = (m + np.log(l))[:, 0]
            pv = p @ np.abs(v)
            # o is sum p' v / sum p' of rounded p' = p (1 + u): off by sum p u (v - o), so by U sum p |v - o| and
            # U sqrt(sum p (v - o)^2) at most
            spread = np.sqrt(np.maximum(p @ (v * v) - o[a:b, hq] ** 2, 0.0))
            err_o = U * (np.abs(o[a:b, hq]) + spread) * 1.01 + 2 * slack * pv + n * W * pv
            tol["o"][a:b, hq] = err_o
            mag = np.where(seen, np.abs(q) @ np.abs(k).T * sc, 0.0).max(1)
            tol["lse"][h, a:b] = 2.0 * d * W * mag + (n + 64) * W + 4 * W * np.abs(lse[h, a:b]) + off
            if dout is None:
                continue
            do = dout[a:b, hq]
            dp = do @ v.T
            D = (do * o[a:b, hq]).sum(1, keepdims=True)
            dc = p * (dp - D)
            ds = dc * slope
            grad[a:b, hv] += p.T @ do
            grad[a:b, hq] = ds @ k * sc
            grad[a:b, hk] += ds.T @ q * sc
            if rest:
                err_o = err_o - U * np.abs(o[a:b, hq]) * 1.01 + 2.0 ** -16 * np.abs(o[a:b, hq])
            err_D = (np.abs(do) * err_o).sum(1, keepdims=True)
            flat = d * W * (np.abs(do) @ np.abs(v).T + np.abs(D))
            err_ds = U * np.abs(ds) * 1.01 + slope * p * (err_D + flat) * (1 + U) + slack * np.abs(ds) + \
                (2.0 ** -20 * np.abs(dc) if cap else 0.0)
            tol["dqkv"][a:b, hv] += U * (p.T @ np.abs(do)) * 1.01 + (slack + n * W) * (p.T @ np.abs(do))
            tol["dqkv"][a:b, hq] = (err_ds @ np.abs(k) + n * W * (np.abs(ds) @ np.abs(k))) * sc
            tol["dqkv"][a:b, hk] += (err_ds.T @ np.abs(q) + n * W * (np.abs(ds).T @ np.abs(q))) * sc
    tol["dqkv"] += U * (np.abs(grad) + tol["dqkv"]) + 1e-30
    return o, lse, grad, tol


def qk_norm_rope(x, lens, first, nq, nkv, d, theta, eps, gq, gk, dy=None):
    """y and, with dy, (dx, dgq, dgk), each with its bounds: (value, bound) pairs.

    Beside one rounding of y and dx: cos and sin good to 2^-22, r to 2^-18 (a sum of d squares, a root, a quotient),
    the sum <a, x> to (d + 16) W of its terms' sizes; the gains' sums of fp32 terms, at most 64 to a lane, to 2^-17."""
    y, ey = x.copy(), np.zeros_like(x)
    dx = None if dy is None else dy.copy()
    ex = np.zeros_like(x)
    dg, eg = [np.zeros(d), np.zeros(d)], [np.zeros(d), np.zeros(d)]
    at = R.bounds_of(lens, first)
    half = d // 2
    freq = theta ** (-2.0 * np.arange(half) / d)

    def turn(v, c, s):
        lo, hi = v[:, :half], v[:, half:]
        return np.concatenate([lo * c - hi * s, lo * s + hi * c], 1)

    def size(v):  # |lo| + |hi| of a pair, for both
        s = np.abs(v[:, :half]) + np.abs(v[:, half:])
        return np.concatenate([s, s], 1)

    for a, b in zip(at, at[1:]):
        ang = np.outer(np.arange(b - a), freq)
        c, s = np.cos(ang), np.sin(ang)
        for h in range(nq + nkv):
            col = slice(h * d, (h + 1) * d)
            g = gq if h < nq else gk
            v = x[a:b, col]
            r = 1.0 / np.sqrt((v * v).mean(1, keepdims=True) + eps)
            n = v * r * g
            y[a:b, col] = turn(n, c, s)
            ey[a:b, col] = U * np.abs(y[a:b, col]) * 1.01 + 2.0 ** -17 * size(n)
            if dy is None:
                continue
            t = dy[a:b, col]
            dn = turn(t, c, -s)
            err_dn = 2.0 ** -20 * size(t)
            dot = (g * dn * v).sum(1, keepdims=True)
            err_dot = ((d + 16) * W * np.abs(g * dn * v) + np.abs(g * v) * err_dn).sum(1, keepdims=True)
            dx[a:b, col] = r * g * dn - v * r ** 3 * dot / d
            flat = 2.0 ** -16 * (np.abs(r * g * dn) + np.abs(v * r ** 3 * dot) / d) + r * np.abs(g) * err_dn + \
                np.abs(v) * r ** 3 * err_dot / d
            ex[a:b, col] = U * np.abs(dx[a:b, col]) * 1.01 + flat * (1 + U)
            k = 0 if h < nq else 1
            dg[k] += (dn * v * r).sum(0)
            eg[k] += (2.0 ** -17 * np.abs(dn * v * r) + err_dn * np.abs(v * r)).sum(0)
    if dy is None:
        return y, ey
    return (y, ey), (dx, ex), (dg[0], eg[0] + 1e-30), (dg[1], eg[1] + 1e-30)
