"""What the losses turn away on the host, before anything is launched.  No GPU: every call below fails its argument checks."""
import ctypes as C
import os
import re

import pytest
import torch

from paper_1901_01544_amd import iwp, losses

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
AT = 0x10000                                              # never dereferenced
S = type("NoStream", (), {"cuda_stream": 0})()
GOOD_CE = dict(h=AT, ld_h=64, w=AT, ld_w=64, tokens=10, dim=64, vocab=100, dtype=1, target=AT, weight=None, scale=1.0, piece=0, loss=AT,
               dh=AT, ld_dh=64, dw=AT, ld_dw=64, dw_dtype=1, ws=AT, bytes=1 << 40)
GOOD_DISTILL = dict(h=AT, ld_h=64, w=AT, ld_w=64, tokens=10, dim=64, vocab=100, dtype=1, index=AT, logit=AT, top=4, temperature=1.0,
                    soft=1.0, target=None, hard=0.0, weight=None, scale=1.0, piece=0, loss=AT, dh=AT, ld_dh=64, dw=AT, ld_dw=64,
                    dw_dtype=1, ws=AT, bytes=1 << 40)
GOOD_BALANCE = dict(x=AT, ld_x=8, tokens=10, experts=8, dtype=0, chosen=AT, slots=2, keep=None, balance=1.0, z=0.0, loss=AT, counts=AT,
                    dx=AT, ld_dx=8, ws=AT, bytes=1 << 30)
NAN, INF = float("nan"), float("inf")
INVALID, ALIGN, WORKSPACE, RANGE = iwp.IWP_EINVAL, iwp.IWP_EALIGN, iwp.IWP_EWORKSPACE, iwp.IWP_ERANGE


def code(call, good, **changed):
    iwp.load()
    args = dict(good, **changed)
    return getattr(iwp._hot(), call)(*args.values(), None)


HEAD = [(dict(h=None), INVALID), (dict(w=None), INVALID), (dict(loss=None), INVALID), (dict(dim=0), INVALID), (dict(vocab=0), INVALID),
        (dict(tokens=(1 << 20) + 1), INVALID), (dict(dim=(1 << 16) + 1, ld_h=1 << 20, ld_w=1 << 20, ld_dh=1 << 20, ld_dw=1 << 20), INVALID),
        (dict(vocab=(1 << 22) + 1), INVALID), (dict(dtype=3), INVALID), (dict(dw_dtype=2), INVALID), (dict(scale=NAN), INVALID),
        (dict(scale=INF), INVALID), (dict(ld_h=63), INVALID), (dict(ld_w=63), INVALID), (dict(ld_dh=63), INVALID), (dict(ld_dw=63), INVALID),
        (dict(ld_h=1 << 23), RANGE), (dict(ld_w=1 << 40), RANGE), (dict(h=AT + 1), ALIGN), (dict(w=AT + 1), ALIGN), (dict(dh=AT + 1), ALIGN),
        (dict(dw=AT + 1), ALIGN), (dict(dw=AT + 2, dw_dtype=0), ALIGN), (dict(loss=AT + 2), ALIGN), (dict(target=AT + 2), ALIGN),
        (dict(weight=AT + 2), ALIGN), (dict(ws=AT + 128), ALIGN), (dict(ws=None), WORKSPACE), (dict(bytes=1000), WORKSPACE)]


@pytest.mark.parametrize("changed,want", HEAD + [(dict(target=None), INVALID)], ids=str)
def test_cross_entropy(changed, want):
    assert code("iwp_head_cross_entropy", GOOD_CE, **changed) == want


@pytest.mark.parametrize("changed,want", HEAD + [
    (dict(index=None), INVALID), (dict(logit=None), INVALID), (dict(top=0), INVALID), (dict(top=1025), INVALID), (dict(temperature=0.0), INVALID),
    (dict(temperature=-1.0), INVALID), (dict(temperature=NAN), INVALID), (dict(temperature=INF), INVALID), (dict(soft=NAN), INVALID),
    (dict(hard=INF), INVALID), (dict(index=AT + 2), ALIGN), (dict(logit=AT + 1), ALIGN)], ids=str)
def test_distill(changed, want):
    assert code("iwp_head_distill", GOOD_DISTILL, **changed) == want


@pytest.mark.parametrize("changed,want", [
    (dict(x=None), INVALID), (dict(chosen=None), INVALID), (dict(loss=None), INVALID), (dict(counts=None), INVALID), (dict(experts=0), INVALID),
    (dict(experts=1025, ld_x=2000, ld_dx=2000), INVALID), (dict(slots=0), INVALID), (dict(slots=9), INVALID), (dict(dtype=3), INVALID),
    (dict(tokens=(1 << 20) + 1), INVALID), (dict(balance=NAN), INVALID), (dict(z=INF), INVALID), (dict(ld_x=7), INVALID), (dict(ld_dx=7), INVALID),
    (dict(x=AT + 2), ALIGN), (dict(dx=AT + 1), ALIGN), (dict(chosen=AT + 2), ALIGN), (dict(loss=AT + 2), ALIGN), (dict(counts=AT + 1), ALIGN),
    (dict(ws=AT + 64), ALIGN), (dict(ws=None), WORKSPACE), (dict(bytes=64), WORKSPACE)], ids=str)
def test_balance(changed, want):
    assert code("iwp_balance", GOOD_BALANCE, **changed) == want


def test_nothing_to_do():
    assert code("iwp_head_cross_entropy", GOOD_CE, tokens=0, h=None, target=None, loss=None, dw=None) == iwp.IWP_OK


def test_workspace_sizes():
    L = iwp.load()
    size = lambda T, D, V, dtype=1, w=AT, ld=None, top=0, piece=0: L.iwp_head_workspace_bytes(T, D, V, dtype, w, ld or D, top, piece)  # noqa: E731
    assert size(10, 64, 100) > 0 and size(0, 64, 100) > 0
    assert 0 == size((1 << 20) + 1, 64, 100) == size(10, 0, 100) == size(10, 64, 0) == size(10, 64, 100, dtype=3) == size(10, 64, 100, top=1025)
    # a piece bounds what the logits take; rows that cannot be read where they lie are copied, binary32 is split
    assert size(8192, 64, 131072) > 8192 * 131072 * 2 > 8 * size(8192, 64, 131072, piece=8192)
    assert size(10, 64, 100000, ld=65) >= size(10, 64, 100000) + 100000 * 64 * 2
    assert size(10, 64, 100000, w=AT + 2) == size(10, 64, 100000, ld=65)
    assert size(10, 64, 100000, dtype=0) >= size(10, 64, 100000) + 100000 * 64 * 4
    assert L.iwp_balance_workspace_bytes(10, 0) == 0 == L.iwp_balance_workspace_bytes(10, 1025) and L.iwp_balance_workspace_bytes(0, 1) > 0


def test_every_declared_loss_is_exported():
    L = iwp.load()
    text = re.sub(r"/\*.*?\*/", "", open(os.path.join(ROOT, "include", "iwp_losses.h")).read(), flags=re.S)
    names = set(re.findall(r"^\s*(?:int|size_t)\s+([a-z][A-Za-z0-9_]*)\s*\(", text, flags=re.M))
    assert {"iwp_head_cross_entropy", "iwp_head_distill", "iwp_balance", "iwp_head_workspace_bytes", "iwp_balance_workspace_bytes"} == names
    at = {name: C.cast(getattr(L, name), C.c_void_p).value for name in iwp._hot().loss_names()}
    assert len(set(at.values())) == len(at) == 3
    with pytest.raises(KeyError):
        iwp._hot().bind_losses({})
    iwp._hot().bind_losses(at)


def test_tensors_that_do_not_fit():
    f = lambda *shape, dtype=torch.bfloat16: torch.empty(*shape, dtype=dtype)  # noqa: E731
    h, w, y, loss = f(4, 8), f(10, 8), f(4, dtype=torch.int32), f(4, dtype=torch.float32)
    with pytest.raises(ValueError, match="device"):
        losses.head_cross_entropy(h, w, y, loss, None, None, None)
    with pytest.raises(ValueError, match="not torch.int32"):
        losses.head_cross_entropy(h.int(), w, y, loss, None, None, None)
    with pytest.raises(ValueError, match="matrices"):
        losses.head_cross_entropy(f(8), w, y, loss, None, None, None)
    with pytest.raises(ValueError, match="device"):
        losses.balance(f(4, 8), f(4, 2, dtype=torch.int32), f(2), f(8), None, None)
    with pytest.raises(ValueError, match="refuses"):
        losses.balance_workspace_bytes(10, 5000)
