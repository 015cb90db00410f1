"""What the calls of post-training refuse, here on the CPU: the library's checks run before any HIP call, the binding's
before the library's."""
from __future__ import annotations

import ctypes

import pytest
import torch

from paper_2510_02483_amd import lib as L
from paper_2510_02483_amd.configs import PackedConfig, ScoreConfig

V = ctypes.c_void_p
C = PackedConfig(total=24, n_seqs=2, n_q_heads=4, n_kv_heads=2, head_dim=64)
A = [V((i + 1) << 36) for i in range(12)]  # disjoint, aligned addresses that nobody reads


def packed(c=C):
    cfg = L.make_packed_cfg(c)
    return ctypes.byref(cfg), L.ls_packed_plan_bytes(C)


def norm_fwd(c=C, theta=1e4, eps=1e-5, plan=A[0], plan_bytes=None, gq=A[1], gk=A[2], src=A[3], dst=A[4]):
    cfg, n = packed(c)
    return L.lib().ls_packed_qk_norm_rope(cfg, plan, n if plan_bytes is None else plan_bytes, theta, eps, gq, gk, src, dst,
                                          None)


def norm_bwd(c=C, theta=1e4, eps=1e-5, plan=A[0], plan_bytes=None, gq=A[1], gk=A[2], src=A[3], dy=A[4], dx=A[5],
             dgq=A[6], dgk=A[7], ws=A[8], ws_bytes=None):
    cfg, n = packed(c)
    need = L.ls_packed_qk_norm_rope_bwd_workspace(C)
    return L.lib().ls_packed_qk_norm_rope_bwd(cfg, plan, n if plan_bytes is None else plan_bytes, theta, eps, gq, gk, src,
                                              dy, dx, dgq, dgk, 0, ws, need if ws_bytes is None else ws_bytes, None)


def at(p, n):
    return V(p.value + n)


@pytest.mark.parametrize("call", [norm_fwd, norm_bwd])
@pytest.mark.parametrize("bad,status", [
    (dict(c=PackedConfig(0, 2, 4, 2, 64)), 2), (dict(c=PackedConfig(24, 2, 4, 3, 64)), 2),
    (dict(c=PackedConfig(24, 2, 4, 2, 100)), 3), (dict(theta=1.0), 2), (dict(theta=float("nan")), 2),
    (dict(eps=-1e-6), 2), (dict(eps=float("nan")), 2), (dict(eps=float("inf")), 2), (dict(plan=None), 1),
    (dict(gq=None), 1), (dict(gk=None), 1), (dict(src=None), 1), (dict(src=at(A[3], 8)), 4), (dict(gk=at(A[2], 2)), 4),
    (dict(plan_bytes=64), 6),
])
def test_qk_norm_refusals(call, bad, status):
    assert call(**bad) == status


@pytest.mark.parametrize("bad,status", [
    (dict(dst=None), 1), (dict(dst=at(A[3], 16)), 5), (dict(dst=A[0]), 5), (dict(dst=A[1]), 5)])
def test_qk_norm_forward_refusals(bad, status):
    assert norm_fwd(**bad) == status


@pytest.mark.parametrize("bad,status", [
    (dict(dx=None), 1), (dict(dy=None), 1), (dict(dx=A[3]), 5), (dict(dx=at(A[4], 16)), 5), (dict(ws=None), 1),
    (dict(ws_bytes=8), 6), (dict(dgq=A[1]), 5), (dict(dgq=A[7]), 5), (dict(dgk=at(A[7], 4)), 4), (dict(ws=A[4]), 5)])
def test_qk_norm_backward_refusals(bad, status):
    assert norm_bwd(**bad) == status


def score_fwd(score, plan_bytes=None, qkv=A[1], o=A[2], lse=A[3], rest=None):
    cfg, n = packed()
    return L.lib().ls_packed_score_attn_fwd(cfg, score, A[0], n if plan_bytes is None else plan_bytes, qkv, o, lse, rest,
                                            None)


def score_bwd(score, plan_bytes=None, qkv=A[1], o=A[2], lse=A[3], dout=A[4], dqkv=A[5], ws=A[6], ws_bytes=None, rest=None):
    cfg, n = packed()
    need = L.ls_packed_attn_bwd_workspace(C)
    return L.lib().ls_packed_score_attn_bwd(cfg, score, A[0], n if plan_bytes is None else plan_bytes, qkv, o, lse, rest,
                                            dout, dqkv, ws, need if ws_bytes is None else ws_bytes, None)


@pytest.mark.parametrize("call", [score_fwd, score_bwd])
@pytest.mark.parametrize("bad,status", [
    (dict(cap=-1.0), 2), (dict(cap=float("nan")), 2), (dict(cap=float("inf")), 3), (dict(cap=0.001), 3),
    (dict(cap=2000.0), 3), (dict(scale=-0.1), 2), (dict(scale=float("nan")), 2), (dict(scale=float("inf")), 2),
    (dict(scale=3e38, cap=0.01), 2), (dict(window=-1), 2)])
def test_score_refusals(call, bad, status):
    sc = L.make_score_cfg(ScoreConfig(**bad))
    assert call(ctypes.byref(sc)) == status


@pytest.mark.parametrize("score", [ScoreConfig(), ScoreConfig(cap=30.0), ScoreConfig(window=5)], ids=["plain", "cap", "window"])
def test_score_attention_refusals(score):
    sc = ctypes.byref(L.make_score_cfg(score))
    assert score_fwd(None) == 1 and score_bwd(None) == 1
    assert score_fwd(sc, plan_bytes=8) == 6 and score_bwd(sc, plan_bytes=8) == 6
    assert score_fwd(sc, qkv=None) == 1 and score_fwd(sc, lse=None) == 1 and score_fwd(sc, o=A[1]) == 5
    assert score_fwd(sc, qkv=at(A[1], 2)) == 4
    assert score_bwd(sc, dqkv=A[1]) == 5 and score_bwd(sc, ws=None) == 1 and score_bwd(sc, ws_bytes=64) == 6
    assert score_bwd(sc, dout=None) == 1
    assert score_fwd(sc, rest=A[2]) == 5 and score_fwd(sc, rest=A[1]) == 5 and score_fwd(sc, rest=at(A[7], 4)) == 4
    assert score_bwd(sc, rest=A[5]) == 5 and score_bwd(sc, rest=at(A[7], 4)) == 4


def tensors(*spec):
    return (L.LsTensor * len(spec))(*[L.LsTensor(*s) for s in spec])


def test_grad_norm_refusals():
    lib, n = L.lib(), L.ls_grad_norm_workspace()
    a, b = 1 << 36, 1 << 37
    ok = tensors((a, 100, 0), (b, 7, 1))
    norm, ws = A[8], A[9]
    assert lib.ls_grad_norm(0, ok, norm, ws, n, None) == 2
    assert lib.ls_grad_norm((1 << 20) + 1, ok, norm, ws, n, None) == 2
    assert lib.ls_grad_norm(2, None, norm, ws, n, None) == 1
    assert lib.ls_grad_norm(2, ok, None, ws, n, None) == 1
    assert lib.ls_grad_norm(2, ok, norm, None, n, None) == 1
    assert lib.ls_grad_norm(2, ok, norm, ws, n - 8, None) == 6
    assert lib.ls_grad_norm(2, ok, V(a + 16), ws, n, None) == 5
    assert lib.ls_grad_norm(2, ok, norm, V(b), n, None) == 5
    for bad, status in (((a, -1, 0), 2), ((a, 1 << 40, 0), 2), ((a, 8, 2), 3), ((None, 8, 0), 1), ((a + 4, 8, 0), 4)):
        assert lib.ls_grad_norm(1, tensors(bad), norm, ws, n, None) == status, bad


def test_grad_clip_refusals():
    lib = L.lib()
    a, b, c = 1 << 36, 1 << 37, 1 << 38
    norm = A[8]

    def clip(grads, out=None, max_norm=1.0, norm=norm):
        return lib.ls_grad_clip(len(grads), tensors(*grads), norm, max_norm, None if out is None else tensors(*out), None)

    ok = [(a, 100, 0), (b, 7, 1)]
    for m in (0.0, -1.0, float("nan"), float("inf")):
        assert clip(ok, max_norm=m) == 2
    assert clip(ok, norm=None) == 1
    assert clip(ok, norm=V(a + 32)) == 5                        # norm inside a tensor that is written
    assert clip([(a, 100, 0), (a, 100, 0)]) == 5                # one tensor twice
    assert clip([(a, 100, 0), (a + 160, 10, 0)]) == 5
    assert clip(ok, [(c, 100, 0), (c + 399 // 16 * 16, 7, 1)]) == 5   # results overlap
    assert clip(ok, [(b, 100, 0), (c, 7, 1)]) == 5              # a result over another's gradient
    assert clip(ok, [(a, 100, 1), (c, 7, 1)]) == 5              # over its own in another type
    assert clip(ok, [(a + 16, 100, 0), (c, 7, 1)]) == 5
    assert clip(ok, [(c, 99, 0), (c + 4096, 7, 1)]) == 2        # another number of elements
    assert clip(ok, [(c, 100, 0), (None, 7, 1)]) == 1
    assert clip(ok, [(c, 100, 5), (c + 4096, 7, 1)]) == 3


def test_binding_of_gradients():
    t = torch.zeros(8)
    for bad in ([], [t.to(torch.float16)], [torch.zeros(8, 8)[:, ::2]], [t]):  # (the last: host memory)
        with pytest.raises(ValueError):
            L.ls_grad_norm(bad, t, t)
        with pytest.raises(ValueError):
            L.ls_grad_clip(bad, t, 1.0)


BF16, F32, U8 = torch.bfloat16, torch.float32, torch.uint8
QKV, O, PLAN, WS, LSE, GAIN = (BF16, (24, 8 * 64)), (BF16, (24, 4 * 64)), (U8, (1 << 14,)), (U8, (1 << 24,)), (F32, (4, 24)), (BF16, (64,))
ENTRIES = {
    "norm": (lambda t: L.ls_packed_qk_norm_rope(C, theta=1e4, eps=1e-5, **t),
             dict(plan=PLAN, q_gain=GAIN, k_gain=GAIN, src=QKV, dst=QKV)),
    "norm_bwd": (lambda t: L.ls_packed_qk_norm_rope_bwd(C, theta=1e4, eps=1e-5, accumulate=False, **t),
                 dict(plan=PLAN, q_gain=GAIN, k_gain=GAIN, src=QKV, dy=QKV, dx=QKV, dq_gain=(F32, (64,)),
                      dk_gain=(F32, (64,)), workspace=WS)),
    "score": (lambda t: L.ls_packed_score_attn_fwd(C, ScoreConfig(cap=5.0), **t), dict(plan=PLAN, qkv=QKV, o=O, lse=LSE, o_rest=O)),
    "score_bwd": (lambda t: L.ls_packed_score_attn_bwd(C, ScoreConfig(cap=5.0), **t),
                  dict(plan=PLAN, qkv=QKV, o=O, lse=LSE, o_rest=O, dout=O, dqkv=QKV, workspace=WS)),
}


@pytest.mark.parametrize("entry,name", [(e, k) for e, (_, spec) in ENTRIES.items() for k in spec])
def test_tensors_that_do_not_fit(entry, name):
    call, spec = ENTRIES[entry]
    good = {k: torch.zeros(shape, dtype=dt) for k, (dt, shape) in spec.items()}
    t = good[name]
    bad = [torch.zeros(2 * t.numel(), dtype=t.dtype)[::2]]
    if name not in ("plan", "workspace"):
        bad += [t.to(torch.float64), t.reshape(-1)[:-1].clone()]
    for b in bad:
        with pytest.raises(ValueError, match=name):
            call(dict(good, **{name: b}))
    with pytest.raises(ValueError, match="GPU"):
        call(good)
