"""Operators of training on packed documents, as timed cases.

Documents of different lengths lie end to end in one row of tokens; rows behind the
last one belong to none.  `cu_seqlens` holds where each document begins, and where the
last one ends.  The operators: rotary positions that restart at every document,
causal grouped-query attention inside each document (forward, and forward with
backward), and the language-model head with its cross-entropy, whose logits are
never kept (the loss alone, and the loss with the gradients of the hidden states and
of the head).  Attention and rotation read a projection buffer whose rows hold the
query heads, then the key heads, then the value heads.

`own` picks between the plain form of each (elementary operations in 32 bits) and
the library's calls.  Values: activations N(0, 1), head weights N(0, 0.02^2), in bf16.
"""
from __future__ import annotations

import math
import random

import torch

own = False

BF16, F32, F64 = torch.bfloat16, torch.float32, torch.float64


def _packed(kind, rows, tail, docs, sigma, nq, nkv, d, docs_seed, **more):
    return dict(kind=kind, rows=rows, tail=tail, docs=docs, sigma=sigma, nq=nq, nkv=nkv, d=d, docs_seed=docs_seed, **more)


def _head(kind, tokens, hidden, vocab, masked):
    return dict(kind=kind, tokens=tokens, hidden=hidden, vocab=vocab, masked=masked)


def listed():
    return [
        # the unit-test sized model's heads on a few short documents: the time of a launch counts
        dict(name="rope_small", **_packed("rope", 253, 6, 5, 0.7, 4, 2, 64, 1, theta=1e4, inverse=False)),
        # a micro-batch of the 3B-shaped block, its four sequences' worth of tokens in documents; the gradients' way back
        dict(name="rope_3b_back", **_packed("rope", 8192, 57, 13, 1.0, 24, 8, 128, 2, theta=5e5, inverse=True)),
        # the unit-test sized model on a row of short documents
        dict(name="attn_fwd_small", **_packed("attn_fwd", 256, 3, 7, 0.9, 4, 2, 64, 3)),
        # evaluation of the 3B-shaped block on documents of very different lengths
        dict(name="attn_fwd_3b", **_packed("attn_fwd", 8192, 57, 13, 1.0, 24, 8, 128, 2)),
        # long context: two documents share the row, heads of the report's 3B model (8 query heads to a kv head)
        dict(name="attn_fwd_long", **_packed("attn_fwd", 16384, 0, 2, 0.5, 16, 2, 128, 4)),
        # training of a small model (12 heads of 64) on documents of odd lengths
        dict(name="attn_train_small", **_packed("attn_train", 1527, 11, 9, 0.8, 12, 4, 64, 5)),
        # training of the 3B-shaped block on a micro-batch of documents
        dict(name="attn_train_3b", **_packed("attn_train", 8192, 57, 13, 1.0, 24, 8, 128, 2)),
        # fine-tuning on short samples, hundreds to a row, multi-head attention
        dict(name="attn_train_short", **_packed("attn_train", 8191, 0, 301, 0.6, 16, 16, 128, 6)),
        # the loss of one token: the head's weights are read once and little else happens
        dict(name="head_loss_one", **_head("head_loss", 1, 2048, 32000, 0.0)),
        # evaluation (perplexity) with the 3B-shaped stack's head
        dict(name="head_loss_3b", **_head("head_loss", 4096, 3072, 128256, 0.002)),
        # training the head on answers only (prompts have no target), odd token count and vocabulary
        dict(name="head_train_small", **_head("head_train", 509, 768, 32003, 0.5)),
        # training the 3B-shaped stack's head on one micro-batch
        dict(name="head_train_3b", **_head("head_train", 8192, 3072, 128256, 0.002)),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    kind = rng.choice(["rope", "attn_fwd", "attn_train", "head_loss", "head_train"])
    if kind.startswith("head"):
        while True:
            c = _head(kind, _log_int(rng, 1, 8192), 8 * _log_int(rng, 16, 512), _log_int(rng, 100, 131072),
                      rng.choice([0.0, 0.01, 0.5]))
            if c["tokens"] * c["hidden"] * c["vocab"] <= 4096 * 3072 * 128256:
                return c
    nkv = rng.choice([1, 2, 4, 8])
    nq = nkv * rng.choice([1, 2, 3, 4, 8])
    rows = _log_int(rng, 1, 8192)
    c = _packed(kind, rows, rng.randrange(0, 1 + rows // 20), 1 + min(rows, 600) * _log_int(rng, 1, 1000) // 1000,
                round(rng.uniform(0.2, 1.5), 2), min(nq, 32), nkv, rng.choice([64, 128]), rng.randrange(1 << 30))
    if kind == "rope":
        c.update(theta=rng.choice([1e4, 5e5]), inverse=rng.random() < 0.5)
    return c


def _lengths(case):
    """The documents' lengths: log-normal shares of the rows; an empty one and one of a single row among four or more."""
    rng, n, left = random.Random(case["docs_seed"]), case["docs"], case["rows"] - case["tail"]
    share = [math.exp(rng.gauss(0.0, case["sigma"])) for _ in range(n)]
    lens = [int(left * s / sum(share)) for s in share]
    if n >= 4:
        lens[1], lens[2] = 0, min(lens[2], 1)
    lens[-1] += left - sum(lens)
    return lens


def _bounds(case):
    at = [0]
    for n in _lengths(case):
        at.append(at[-1] + n)
    return at


def prepare(case, seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)

    def normal(*shape, std=1.0):
        return (torch.randn(*shape, generator=g, device="cuda", dtype=F32) * std).to(BF16)

    s = {"case": case}
    if case["kind"].startswith("head"):
        t, h, v = case["tokens"], case["hidden"], case["vocab"]
        s["h"], s["embed"] = normal(t, h), normal(v, h, std=0.02)
        target = torch.randint(0, v, (t,), generator=g, device="cuda", dtype=torch.int32)
        without = torch.rand(t, generator=g, device="cuda") < case["masked"]
        s["targets"] = torch.where(without, torch.full_like(target, -1), target)
        # one of four micro-batches that are accumulated
        s["dloss"] = torch.full((1,), 0.25, dtype=F32, device="cuda")
    else:
        rows, nq, nkv, d = case["rows"], case["nq"], case["nkv"], case["d"]
        s["cu_seqlens"] = torch.tensor(_bounds(case), dtype=torch.int32, device="cuda")
        s["qkv"] = normal(rows, (nq + 2 * nkv) * d)
        if case["kind"] == "attn_train":
            s["dout"] = normal(rows, nq * d)
    if own:
        _buffers(s)
    return s


def _buffers(s):
    """Outputs and workspaces, made once as a training program does."""
    from paper_2510_02483_amd import lib
    from paper_2510_02483_amd.configs import PackedConfig

    c = s["case"]
    if c["kind"].startswith("head"):
        t, h, v = c["tokens"], c["hidden"], c["vocab"]
        s["loss"] = torch.zeros(1, dtype=F32, device="cuda")
        s["row_loss"] = torch.zeros(t, dtype=F32, device="cuda")
        s["lse"] = torch.zeros(t, dtype=F32, device="cuda")
        s["workspace"] = torch.empty(lib.ls_head_loss_workspace(t, h, v), dtype=torch.uint8, device="cuda")
        if c["kind"] == "head_train":
            s["dh"] = torch.zeros(t, h, dtype=BF16, device="cuda")
            s["d_embed"] = torch.zeros(v, h, dtype=BF16, device="cuda")
        return
    cfg = s["cfg"] = PackedConfig(total=c["rows"], n_seqs=c["docs"], n_q_heads=c["nq"], n_kv_heads=c["nkv"],
                                  head_dim=c["d"])
    s["plan"] = torch.empty(lib.ls_packed_plan_bytes(cfg), dtype=torch.uint8, device="cuda")
    if c["kind"] == "rope":
        s["out"] = torch.zeros_like(s["qkv"])
        return
    s["o"] = torch.zeros(c["rows"], c["nq"] * c["d"], dtype=BF16, device="cuda")
    s["lse"] = torch.zeros(c["nq"], c["rows"], dtype=F32, device="cuda")
    if c["kind"] == "attn_train":
        s["dqkv"] = torch.zeros_like(s["qkv"])
        s["workspace"] = torch.empty(lib.ls_packed_attn_bwd_workspace(cfg), dtype=torch.uint8, device="cuda")


def run(s):
    return _run_own(s) if own else _run_plain(s)


def _run_own(s):
    from paper_2510_02483_amd import lib

    c = s["case"]
    if c["kind"].startswith("head"):
        lib.ls_head_loss_fwd(s["h"], s["embed"], s["targets"], s["loss"], s["row_loss"], s["lse"], s["workspace"])
        out = {"loss": s["loss"], "row_loss": s["row_loss"], "lse": s["lse"]}
        if c["kind"] == "head_train":
            lib.ls_head_loss_bwd(s["h"], s["embed"], s["targets"], s["lse"], s["dloss"], s["dh"], s["d_embed"], False,
                                 s["workspace"])
            out.update(dh=s["dh"], d_embed=s["d_embed"])
        return out
    # the plan belongs to the batch's documents: every layer uses it; here one layer pays for it
    lib.ls_packed_plan(s["cfg"], s["cu_seqlens"], s["plan"])
    if c["kind"] == "rope":
        lib.ls_packed_rope(s["cfg"], s["plan"], c["theta"], s["qkv"], s["out"], inverse=c["inverse"])
        return {"qkv": s["out"]}
    lib.ls_packed_attn_fwd(s["cfg"], s["plan"], s["qkv"], s["o"], s["lse"])
    out = {"o": s["o"], "lse": s["lse"]}
    if c["kind"] == "attn_train":
        lib.ls_packed_attn_bwd(s["cfg"], s["plan"], s["qkv"], s["o"], s["lse"], s["dout"], s["dqkv"], s["workspace"])
        out["dqkv"] = s["dqkv"]
    return out


# ---- plain forms: elementary operations in 32 bits, over all rows at once ---------------


def _documents(s):
    """Of every row: the first row of its document, and whether it has one."""
    cu = s["cu_seqlens"]
    row = torch.arange(s["case"]["rows"], device="cuda")
    doc = (row[:, None] >= cu[None, :]).sum(1) - 1
    inside = doc < cu.numel() - 1
    return row, cu.long()[doc.clamp(max=cu.numel() - 2)], inside


def _run_plain(s):
    kind = s["case"]["kind"]
    if kind.startswith("head"):
        return _plain_head(s)
    return _plain_rope(s) if kind == "rope" else _plain_attention(s)


def _plain_rope(s):
    c = s["case"]
    row, start, inside = _documents(s)
    half = c["d"] // 2
    turned = c["nq"] + c["nkv"]
    # angles of far positions lose their fraction in 32 bits
    freq = float(c["theta"]) ** (-torch.arange(half, device="cuda", dtype=F64) / half)
    angle = (row - start).to(F64)[:, None, None] * freq
    cos, sin = angle.cos().float(), angle.sin().float()
    if c["inverse"]:
        sin = -sin
    x = s["qkv"].float().view(c["rows"], -1, 2, half)
    a, b = x[:, :turned, 0], x[:, :turned, 1]
    out = x.clone()
    out[:, :turned, 0] = a * cos - b * sin
    out[:, :turned, 1] = a * sin + b * cos
    out = torch.where(inside[:, None, None, None], out, torch.zeros_like(out))
    return {"qkv": out.view(c["rows"], -1).to(BF16)}


def _plain_attention(s):
    c = s["case"]
    rows, nq, nkv, d = c["rows"], c["nq"], c["nkv"], c["d"]
    group = nq // nkv
    row, start, inside = _documents(s)
    seen = (row[None, :] >= start[:, None]) & (row[None, :] <= row[:, None]) & inside[:, None] & inside[None, :]

    def heads(x, n):  # [rows, n * d] -> [nkv, n / nkv, rows, d], contiguous
        return x.float().view(rows, nkv, n // nkv, d).permute(1, 2, 0, 3).contiguous()

    def back(x):  # and back
        return x.permute(2, 0, 1, 3).reshape(rows, -1)

    q, k, v = s["qkv"].split([nq * d, nkv * d, nkv * d], dim=1)
    q, k, v = heads(q, nq), heads(k, nkv), heads(v, nkv)
    scale = 1.0 / math.sqrt(d)
    p = torch.matmul(q * scale, k.transpose(-1, -2))
    p = torch.where(seen, p, torch.full_like(p, -math.inf))
    top = p.amax(-1, keepdim=True)
    top = torch.where(inside[:, None], top, torch.zeros_like(top))
    p = torch.exp(p - top)
    total = p.sum(-1, keepdim=True)
    total = torch.where(inside[:, None], total, torch.ones_like(total))
    p = p / total
    o = torch.matmul(p, v)
    lse = torch.where(inside, (top + torch.log(total)).reshape(nq, rows), torch.zeros(1, device="cuda"))
    out = {"o": back(o).to(BF16), "lse": lse}
    if c["kind"] == "attn_train":
        do = heads(s["dout"], nq)
        do = torch.where(inside[:, None], do, torch.zeros_like(do))
        dv = torch.matmul(p.transpose(-1, -2), do).sum(1, keepdim=True)
        ds = torch.matmul(do, v.transpose(-1, -2))
        ds = p * (ds - (do * o).sum(-1, keepdim=True)) * scale
        dq = torch.matmul(ds, k)
        dk = torch.matmul(ds.transpose(-1, -2), q).sum(1, keepdim=True)
        out["dqkv"] = torch.cat([back(dq), back(dk), back(dv)], dim=1).to(BF16)
    return out


def _plain_head(s):
    h, e, target = s["h"].float(), s["embed"].float(), s["targets"].long()
    z = torch.matmul(h, e.t())
    top = z.amax(1, keepdim=True)
    p = torch.exp(z - top)
    total = p.sum(1, keepdim=True)
    lse = (top + torch.log(total)).view(-1)
    has = target >= 0
    at = target.clamp(min=0)
    row_loss = torch.where(has, lse - z[torch.arange(at.numel(), device="cuda"), at], torch.zeros_like(lse))
    count = has.sum().clamp(min=1).float()
    out = {"loss": (row_loss.double().sum() / count.double()).float().view(1), "row_loss": row_loss, "lse": lse}
    if s["case"]["kind"] == "head_train":
        del z
        dz = p / total
        dz[torch.arange(at.numel(), device="cuda"), at] -= 1.0
        dz = dz * (has.float() * (s["dloss"] / count))[:, None]
        out["dh"] = torch.matmul(dz, e).to(BF16)
        out["d_embed"] = torch.matmul(dz.t(), h).to(BF16)
    return out


def work(case):
    if case["kind"].startswith("head"):
        t, h, v = case["tokens"], case["hidden"], case["vocab"]
        size = 2 * (t * h + v * h) + 4 * t + 4 + 8 * t
        if case["kind"] == "head_loss":
            return {"bytes": size, "flops": 2 * t * h * v}
        return {"bytes": size + 2 * (t * h + v * h) + 4, "flops": 6 * t * h * v}
    nq, nkv, d = case["nq"], case["nkv"], case["d"]
    lens = _lengths(case)
    rows = sum(lens)
    qkv, o, cu = rows * (nq + 2 * nkv) * d * 2, rows * nq * d * 2, 4 * (len(lens) + 1)
    if case["kind"] == "rope":
        return {"bytes": 2 * qkv + cu, "flops": 3 * rows * (nq + nkv) * d}
    pairs = sum(n * (n + 1) // 2 for n in lens) * nq * d
    if case["kind"] == "attn_fwd":
        return {"bytes": qkv + o + 4 * rows * nq + cu, "flops": 4 * pairs}
    return {"bytes": 2 * qkv + 2 * o + 4 * rows * nq + cu, "flops": 14 * pairs}


# ---- the definitions in 64 bits, document by document ------------------------------------


def exact(case, seed):
    s = prepare(case, seed)
    if case["kind"].startswith("head"):
        return _exact_head(s)
    at = _bounds(case)
    spans = [(a, b) for a, b in zip(at, at[1:]) if b > a]
    return _exact_rope(s, spans) if case["kind"] == "rope" else _exact_attention(s, spans)


def _exact_rope(s, spans):
    c, d = s["case"], s["case"]["d"]
    out = torch.zeros(s["qkv"].shape, dtype=F64, device="cuda")
    sign = -1.0 if c["inverse"] else 1.0
    omega = torch.tensor([math.pow(c["theta"], -2.0 * i / d) for i in range(d // 2)], dtype=F64, device="cuda")
    for a, b in spans:
        turn = torch.polar(torch.ones(b - a, d // 2, dtype=F64, device="cuda"),
                           sign * torch.outer(torch.arange(b - a, dtype=F64, device="cuda"), omega))
        out[a:b] = s["qkv"][a:b].double()
        for head in range(c["nq"] + c["nkv"]):
            part = out[a:b, head * d:(head + 1) * d]
            z = torch.complex(part[:, :d // 2].contiguous(), part[:, d // 2:].contiguous()) * turn
            part[:, :d // 2], part[:, d // 2:] = z.real, z.imag
    return {"qkv": out}


def _exact_attention(s, spans):
    c = s["case"]
    rows, nq, nkv, d = c["rows"], c["nq"], c["nkv"], c["d"]
    x = s["qkv"].double()
    o = torch.zeros(rows, nq * d, dtype=F64, device="cuda")
    lse = torch.zeros(nq, rows, dtype=F64, device="cuda")
    train = c["kind"] == "attn_train"
    grad = torch.zeros(x.shape, dtype=F64, device="cuda")
    for a, b in spans:
        n = b - a
        future = torch.triu(torch.ones(n, n, dtype=torch.bool, device="cuda"), 1)
        for i in range(nq):
            j = i // (nq // nkv)
            qs, ks = slice(i * d, (i + 1) * d), slice((nq + j) * d, (nq + j + 1) * d)
            vs = slice((nq + nkv + j) * d, (nq + nkv + j + 1) * d)
            q, k, v = x[a:b, qs], x[a:b, ks], x[a:b, vs]
            score = (q @ k.T / math.sqrt(d)).masked_fill(future, -math.inf)
            norm = torch.logsumexp(score, 1)
            p = torch.exp(score - norm[:, None])
            o[a:b, qs] = p @ v
            lse[i, a:b] = norm
            if train:
                do = s["dout"][a:b, qs].double()
                grad[a:b, vs] += p.T @ do
                dp = do @ v.T
                ds = p * (dp - (p * dp).sum(1, keepdim=True)) / math.sqrt(d)
                grad[a:b, qs] = ds @ k
                grad[a:b, ks] += ds.T @ q
    out = {"o": o, "lse": lse}
    if train:
        out["dqkv"] = grad
    return out


def _exact_head(s):
    """Blocks of rows, so that the 64-bit logits stay small."""
    t, h = s["h"].shape
    train = s["case"]["kind"] == "head_train"
    e = s["embed"].double()
    valid = (s["targets"] >= 0)
    n = max(int(valid.sum()), 1)
    lse, row_loss = torch.empty(t, dtype=F64, device="cuda"), torch.zeros(t, dtype=F64, device="cuda")
    dh, de = torch.zeros(t, h, dtype=F64, device="cuda"), torch.zeros(e.shape, dtype=F64, device="cuda")
    for a in range(0, t, 1024):
        x = s["h"][a:a + 1024].double()
        z = x @ e.T
        lse[a:a + 1024] = torch.logsumexp(z, 1)
        which = valid[a:a + 1024].nonzero().view(-1)
        goal = s["targets"][a:a + 1024][which].long()
        row_loss[a + which] = lse[a + which] - z[which, goal]
        if train:
            dz = torch.zeros_like(z)
            dz[which] = torch.exp(z[which] - lse[a + which][:, None])
            dz[which, goal] -= 1.0
            dz *= s["dloss"].double() / n
            dh[a:a + 1024] = dz @ e
            de += dz.T @ x
    out = {"loss": (row_loss.sum() / n).view(1), "row_loss": row_loss, "lse": lse}
    if train:
        out.update(dh=dh, d_embed=de)
    return out
