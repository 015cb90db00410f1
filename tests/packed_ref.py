"""Packed sequences in 64 bits, from the definitions, and how far the kernels may be from them.

Every bound counts roundings: u = 2^-8 is the largest relative error of one
rounding to bf16, W = 2^-24 that of one fp32 operation."""
from __future__ import annotations

import numpy as np

U = 2.0 ** -8
W = 2.0 ** -24


def bounds_of(lens, first=0):
    return np.concatenate([[first], first + np.cumsum(lens)]).astype(np.int64)


def rope(x, lens, first, nq, nkv, d, theta, inverse=False):
    """x [total, (nq + 2 nkv) d] -> the same with q and k turned (float64)."""
    out = x.copy()
    at = bounds_of(lens, first)
    i = np.arange(d // 2)
    for a, b in zip(at, at[1:]):
        ang = np.outer(np.arange(b - a), theta ** (-2.0 * i / d)) * (-1.0 if inverse else 1.0)
        c, s = np.cos(ang), np.sin(ang)
        for h in range(nq + nkv):
            lo, hi = x[a:b, h * d:h * d + d // 2], x[a:b, h * d + d // 2:(h + 1) * d]
            out[a:b, h * d:h * d + d // 2] = lo * c - hi * s
            out[a:b, h * d + d // 2:(h + 1) * d] = lo * s + hi * c
    return out


def attention(qkv, lens, first, nq, nkv, d, dout=None):
    """o, lse (and dqkv) of the packed sequences, and elementwise bounds of the kernels' error.

    Forward: the probabilities are rounded to bf16 for their product with v, and o
    once more: |err o| <= u (|o| + sum p |v|).  The log-sum-exp stays in fp32: its
    scores are sums of d products, its sum has at most n terms.
    Backward: p is rounded for dv, dS = p (dP - D) for dq and dk, D comes from the
    rounded o: |err D| <= sum |dO| |err o|.  fp32 slack: W per term of every sum
    and 2^-18 relative on p (the exponent's fp32 error at |score| up to 2^5)."""
    total = qkv.shape[0]
    o = np.zeros((total, nq * d))
    lse = np.zeros((nq, total))
    grad = np.zeros_like(qkv)
    tol = {"o": np.zeros_like(o), "lse": np.zeros_like(lse), "dqkv": np.zeros_like(qkv)}
    at = bounds_of(lens, first)
    sc = 1.0 / np.sqrt(d)
    slack = 2.0 ** -18
    for a, b in zip(at, at[1:]):
        n = int(b - a)
        if n == 0:
            continue
        causal = np.tril(np.ones((n, n), bool))
        for h in range(nq):
            g = h // (nq // nkv)
            hq, hk, hv = (slice(x * d, (x + 1) * d) for x in (h, nq + g, nq + nkv + g))
            q, k, v = qkv[a:b, hq], qkv[a:b, hk], qkv[a:b, hv]
            s = np.where(causal, q @ k.T * sc, -np.inf)
            m = s.max(1, keepdims=True)
            e = np.exp(s - m)
            l = e.sum(1, keepdims=True)
            p = e / l
            o[a:b, hq] = p @ v
            lse[h, a:b] = (m + np.log(l))[:, 0]
            pv = p @ np.abs(v)
            err_o = U * (np.abs(o[a:b, hq]) + pv) * 1.01 + slack * pv + n * W * pv
            tol["o"][a:b, hq] = err_o
            mag = np.where(causal, np.abs(q) @ np.abs(k).T * sc, 0.0).max(1)
            tol["lse"][h, a:b] = 2.0 * d * W * mag + (n + 64) * W + 4 * W * np.abs(lse[h, a:b])
            if dout is None:
                continue
            do = dout[a:b, hq]
            dp = do @ v.T
            D = (do * o[a:b, hq]).sum(1, keepdims=True)
            ds = p * (dp - D)
            grad[a:b, hv] += p.T @ do
            grad[a:b, hq] = ds @ k * sc
            grad[a:b, hk] += ds.T @ q * sc
            err_D = (np.abs(do) * err_o).sum(1, keepdims=True)
            # dP and D are fp32 sums of d terms, D and dP of similar size cancel
            flat = d * W * (np.abs(do) @ np.abs(v).T + np.abs(D))
            err_ds = U * np.abs(ds) * 1.01 + p * (err_D + flat) * (1 + U) + slack * np.abs(ds)
            tol["dqkv"][a:b, hv] += U * (p.T @ np.abs(do)) * 1.01 + (slack + n * W) * (p.T @ np.abs(do))
            tol["dqkv"][a:b, hq] = (err_ds @ np.abs(k) + n * W * (np.abs(ds) @ np.abs(k))) * sc
            tol["dqkv"][a:b, hk] += (err_ds.T @ np.abs(q) + n * W * (np.abs(ds).T @ np.abs(q))) * sc
    tol["dqkv"] += U * (np.abs(grad) + tol["dqkv"]) + 1e-30
    return o, lse, grad, tol
