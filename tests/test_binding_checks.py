"""Tensors that the calls of packed sequences and of the head loss cannot take: the library sees addresses only, so the
binding refuses another type, another number of elements, gaps, and memory that is not the current GPU's.  No call
here gets as far as the library."""
from __future__ import annotations

import pytest
import torch

from paper_2510_02483_amd import lib as L
from paper_2510_02483_amd.configs import PackedConfig

BF16, F32, I32, U8 = torch.bfloat16, torch.float32, torch.int32, torch.uint8
C = PackedConfig(total=24, n_seqs=2, n_q_heads=4, n_kv_heads=2, head_dim=64)
T, H, V = 6, 16, 40


def packed(name):
    qkv, o = (BF16, (24, 8 * 64)), (BF16, (24, 4 * 64))
    plan, lse, ws = (U8, (1 << 14,)), (F32, (4, 24)), (U8, (1 << 24,))
    return {
        "plan": (lambda t: L.ls_packed_plan(C, **t), dict(cu_seqlens=(I32, (3,)), plan=plan)),
        "rope": (lambda t: L.ls_packed_rope(C, theta=1e4, **t), dict(plan=plan, src=qkv, dst=qkv)),
        "fwd": (lambda t: L.ls_packed_attn_fwd(C, **t), dict(plan=plan, qkv=qkv, o=o, lse=lse)),
        "bwd": (lambda t: L.ls_packed_attn_bwd(C, **t),
                dict(plan=plan, qkv=qkv, o=o, lse=lse, dout=o, dqkv=qkv, workspace=ws)),
    }[name]


def head(name):
    common = dict(h=(BF16, (T, H)), embed=(BF16, (V, H)), targets=(I32, (T,)), lse=(F32, (T,)), workspace=(U8, (1 << 20,)))
    grads = dict(common, dloss=(F32, (1,)), dh=(BF16, (T, H)))

    def bwd(t):
        L.ls_head_loss_bwd(accumulate=False, **t)

    return {
        "loss": (lambda t: L.ls_head_loss_fwd(**t), dict(common, loss=(F32, (1,)), row_loss=(F32, (T,)))),
        "grads": (bwd, dict(grads, d_embed=(F32, (V, H)))),
        "grads_bf16": (bwd, dict(grads, d_embed=(BF16, (V, H)))),
    }[name]


ENTRIES = {n: packed(n) for n in ("plan", "rope", "fwd", "bwd")} | {n: head(n) for n in ("loss", "grads", "grads_bf16")}
ANY_BYTES = ("plan", "workspace")  # of any type; their size is the library's to check


def tensors(spec):
    return {k: torch.zeros(shape, dtype=dt) for k, (dt, shape) in spec.items()}


def with_gaps(t):
    return torch.zeros(2 * t.numel(), dtype=t.dtype)[::2].view(t.shape) if t.dim() == 1 else \
        torch.zeros(t.shape[0], 2 * t.shape[1], dtype=t.dtype)[:, ::2]


CASES = [(e, k) for e, (_, spec) in ENTRIES.items() for k in spec]


@pytest.mark.parametrize("entry,name", CASES)
def test_another_type_number_or_stride(entry, name):
    call, spec = ENTRIES[entry]
    good = tensors(spec)[name]
    bad = [with_gaps(good)] if good.numel() > 1 else []
    if name not in ANY_BYTES:
        bad += [good.to(torch.float16), good.to(torch.float64), good[:-1].clone()]
        if good.dtype is I32:
            bad.append(torch.cat([good, good]))
        if good.dim() == 2:
            bad.append(good[:, :-8].contiguous())
    for t in bad:
        # (a longer or shorter h or embed makes the others' sizes wrong)
        said = name if good.dim() == 1 or name not in ("h", "embed") else "must"
        with pytest.raises(ValueError, match=said):
            call(dict(tensors(spec), **{name: t}))


@pytest.mark.parametrize("entry,name", CASES)
def test_a_longer_buffer_is_taken(entry, name):
    """A buffer made for the longest batch: the call gets as far as the check of the device."""
    call, spec = ENTRIES[entry]
    good = tensors(spec)[name]
    if good.dtype is I32 or name in ("h", "embed"):  # (their shape is the problem's)
        return
    with pytest.raises(ValueError, match="GPU"):
        call(dict(tensors(spec), **{name: torch.cat([good, good])}))


@pytest.mark.parametrize("entry", ENTRIES)
def test_host_memory(entry):
    call, spec = ENTRIES[entry]
    with pytest.raises(ValueError, match="GPU"):
        call(tensors(spec))


def test_a_gradient_of_neither_type():
    """A half-precision d_embed has half the bytes that the library would write."""
    call, spec = ENTRIES["grads"]
    with pytest.raises(ValueError, match="d_embed"):
        call(dict(tensors(spec), d_embed=torch.zeros(V, H, dtype=torch.float16)))


@pytest.mark.parametrize("entry", ["loss", "grads"])
def test_head_weights_of_another_width(entry):
    call, spec = ENTRIES[entry]
    with pytest.raises(ValueError, match="embed"):
        call(dict(tensors(spec), embed=torch.zeros(V, H - 8, dtype=BF16)))
