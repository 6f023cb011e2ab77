"""What the routed layer's operators and the clipping turn away on the host, before anything is launched.  No GPU: every call below fails its
argument checks or has nothing to do."""
import ctypes as C
import os
import re

import pytest
import torch

from paper_1901_01544_amd import clipping, experts, iwp

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
AT = 0x10000                                              # never dereferenced
GOOD_ROUTE = dict(x=AT, ld_x=16, tokens=10, experts=16, dtype=0, bias=None, scores=0, groups=4, top_groups=2, group_top=2, renormalise=0, scale=1.0,
                  keep=None, chosen=AT, weight=AT, slots=4)
GOOD_GRADIENT = dict(x=AT, ld_x=16, tokens=10, experts=16, dtype=1, chosen=AT, dweight=AT, slots=4, scores=0, renormalise=0, scale=1.0, keep=None,
                     plus=AT, ld_plus=16, dx=AT, ld_dx=16)
GOOD_PRODUCT = dict(x=AT, ld_x=64, by_slot=0, w=AT, ld_w=64, step_w=2048, tokens=100, slots=2, experts=4, width=64, out=32, dtype=1, chosen=AT, y=AT,
                    ld_y=32, ws=AT, bytes=1 << 40)
GOOD_BACK = dict(x=AT, ld_x=64, by_slot=0, w=AT, ld_w=64, step_w=2048, tokens=10, slots=2, experts=4, width=64, out=32, dtype=1, chosen=AT, dy=AT,
                 ld_dy=32, dx=AT, ld_dx=64, dw=AT, ld_dw=64, step_dw=2048, dw_dtype=0, ws=AT, bytes=1 << 40)
NAN, INF = float("nan"), float("inf")
INVALID, ALIGN, WORKSPACE, RANGE = iwp.IWP_EINVAL, iwp.IWP_EALIGN, iwp.IWP_EWORKSPACE, iwp.IWP_ERANGE


def code(call, good, **changed):
    iwp.load()
    return getattr(iwp._hot(), call)(*dict(good, **changed).values(), None)


@pytest.mark.parametrize("changed,want", [
    (dict(x=None), INVALID), (dict(chosen=None), INVALID), (dict(weight=None), INVALID), (dict(experts=0), INVALID),
    (dict(experts=1028, ld_x=2000), INVALID), (dict(tokens=(1 << 20) + 1), INVALID), (dict(dtype=3), INVALID), (dict(scores=2), INVALID),
    (dict(renormalise=2), INVALID), (dict(groups=0), INVALID), (dict(groups=3), INVALID), (dict(top_groups=0), INVALID), (dict(top_groups=5), INVALID),
    (dict(group_top=0), INVALID), (dict(group_top=3), INVALID), (dict(groups=16, group_top=2), INVALID), (dict(slots=0), INVALID), (dict(slots=9), INVALID),
    (dict(scale=NAN), INVALID), (dict(scale=INF), INVALID), (dict(ld_x=15), INVALID), (dict(ld_x=-16), INVALID), (dict(x=AT + 2), ALIGN),
    (dict(x=AT + 1, dtype=1), ALIGN), (dict(bias=AT + 2), ALIGN), (dict(chosen=AT + 2), ALIGN), (dict(weight=AT + 1), ALIGN),
    (dict(tokens=0, x=None, chosen=None, weight=None), iwp.IWP_OK)], ids=str)
def test_route(changed, want):
    assert code("iwp_route", GOOD_ROUTE, **changed) == want


@pytest.mark.parametrize("changed,want", [
    (dict(x=None), INVALID), (dict(chosen=None), INVALID), (dict(dweight=None), INVALID), (dict(dx=None), INVALID), (dict(experts=0), INVALID),
    (dict(experts=1028, ld_x=2000, ld_dx=2000, ld_plus=2000), INVALID), (dict(tokens=(1 << 20) + 1), INVALID), (dict(dtype=3), INVALID),
    (dict(scores=2), INVALID), (dict(renormalise=2), INVALID), (dict(slots=0), INVALID), (dict(slots=17), INVALID), (dict(scale=NAN), INVALID),
    (dict(ld_x=15), INVALID), (dict(ld_dx=15), INVALID), (dict(ld_plus=15), INVALID), (dict(x=AT + 1), ALIGN), (dict(dx=AT + 1), ALIGN),
    (dict(plus=AT + 1), ALIGN), (dict(chosen=AT + 2), ALIGN), (dict(dweight=AT + 2), ALIGN),
    (dict(tokens=0, x=None, chosen=None, dweight=None, dx=None), iwp.IWP_OK)], ids=str)
def test_route_gradient(changed, want):
    assert code("iwp_route_gradient", GOOD_GRADIENT, **changed) == want


PRODUCTS = [
    (dict(x=None), INVALID), (dict(w=None), INVALID), (dict(chosen=None), INVALID), (dict(by_slot=2), INVALID), (dict(slots=0), INVALID), (dict(slots=5), INVALID),
    (dict(experts=0), INVALID), (dict(experts=1025), INVALID), (dict(width=0), INVALID), (dict(out=0), INVALID), (dict(dtype=3), INVALID),
    (dict(width=(1 << 16) + 1), INVALID), (dict(out=(1 << 16) + 1), INVALID), (dict(tokens=(1 << 20) + 1), INVALID),
    (dict(tokens=1 << 20, slots=17, experts=17), INVALID), (dict(ld_x=63), INVALID), (dict(ld_w=63), INVALID), (dict(step_w=2047), INVALID),
    (dict(step_w=-2048), INVALID), (dict(ld_x=1 << 23), RANGE), (dict(ld_w=1 << 23, step_w=1 << 40), RANGE),
    (dict(ld_x=1 << 22, ld_w=1 << 22, step_w=1 << 40, dtype=0, dw_dtype=0), RANGE), (dict(x=AT + 1), ALIGN), (dict(w=AT + 1), ALIGN), (dict(chosen=AT + 2), ALIGN),
    (dict(ws=AT + 128), ALIGN), (dict(ws=None), WORKSPACE), (dict(bytes=1000), WORKSPACE)]


@pytest.mark.parametrize("changed,want", PRODUCTS + [(dict(y=None), INVALID), (dict(ld_y=31), INVALID), (dict(ld_y=1 << 23), RANGE), (dict(y=AT + 1), ALIGN),
                                                     (dict(tokens=0, x=None, chosen=None, y=None, ws=None, bytes=0), iwp.IWP_OK)], ids=str)
def test_product(changed, want):
    assert code("iwp_expert_product", GOOD_PRODUCT, **{k: v for k, v in changed.items() if k != "dw_dtype"}) == want


@pytest.mark.parametrize("changed,want", PRODUCTS + [
    (dict(dy=None), INVALID), (dict(ld_dy=31), INVALID), (dict(ld_dx=63), INVALID), (dict(ld_dw=63), INVALID), (dict(step_dw=2047), INVALID), (dict(dw_dtype=2), INVALID),
    (dict(ld_dy=1 << 23), RANGE), (dict(ld_dx=1 << 23), RANGE), (dict(ld_dw=1 << 22, step_dw=1 << 40), RANGE), (dict(dy=AT + 1), ALIGN), (dict(dx=AT + 1), ALIGN),
    (dict(dw=AT + 2), ALIGN), (dict(dx=None, dw=None, ws=None, bytes=0), iwp.IWP_OK), (dict(tokens=0, x=None, chosen=None, dy=None, dw=None, ws=None), iwp.IWP_OK)], ids=str)
def test_product_gradient(changed, want):
    assert code("iwp_expert_product_gradient", GOOD_BACK, **changed) == want


def test_workspace_sizes():
    L = iwp.load()

    def size(tokens=100, slots=2, experts=8, width=64, out=32, dtype=1, w=AT, ld=None, step=None, by_slot=0, gradient=0):
        return L.iwp_expert_product_workspace_bytes(tokens, slots, experts, width, out, dtype, w, ld or width, step or out * (ld or width), by_slot, gradient)

    assert size() > 0 and size(tokens=0) > 0 and size(gradient=1) > size()
    assert 0 == size(slots=9) == size(tokens=(1 << 20) + 1) == size(experts=0) == size(width=0) == size(out=0) == size(dtype=3) == size(experts=1025)
    # matrices that cannot be read by 16 bytes where they lie are copied
    many = dict(tokens=1000, experts=64, width=1000, out=1000)
    for other in (dict(w=AT + 2), dict(ld=1001), dict(width=1001), dict(step=1000 * 1000 + 4)):
        assert size(**dict(many, **other)) >= size(**many) + 64 * 1000 * 1000 * 2
    assert size(gradient=1, tokens=4096) > size(gradient=1, tokens=4096, by_slot=1)
    # few rows need none; sizes that no launch takes are refused by the calls too
    assert size(tokens=4, width=1001, out=1000, experts=64) == 256
    assert size(tokens=1 << 20, slots=16, experts=16, width=1 << 16) == 0
    assert code("iwp_expert_product", GOOD_PRODUCT, tokens=1 << 20, slots=16, experts=16, width=1 << 16, ld_x=1 << 16, ld_w=1 << 16, step_w=1 << 30) == INVALID


def test_every_declared_call_is_exported():
    L = iwp.load()
    names = set()
    for header in ("iwp_experts.h", "iwp_clip.h"):
        text = re.sub(r"/\*.*?\*/", "", open(os.path.join(ROOT, "include", header)).read(), flags=re.S)
        names |= set(re.findall(r"^\s*(?:int|size_t|void)\s+([a-z][A-Za-z0-9_]*)\s*\(", text, flags=re.M))
    assert all(hasattr(L, name) for name in names)
    hot = set(iwp._hot().layer_names())
    assert hot <= names and "iwp_clip" in hot and "iwp_route" in hot
    at = {name: C.cast(getattr(L, name), C.c_void_p).value for name in hot}
    assert len(set(at.values())) == len(at)
    with pytest.raises(KeyError):
        iwp._hot().bind_layers({})
    iwp._hot().bind_layers(at)


def test_tensors_that_do_not_fit():
    f = lambda *shape, dtype=torch.bfloat16: torch.empty(*shape, dtype=dtype)  # noqa: E731
    x, chosen, weight = f(4, 8), f(4, 2, dtype=torch.int32), f(4, 2, dtype=torch.float32)
    with pytest.raises(ValueError, match="device"):
        experts.route(x, chosen, weight)
    with pytest.raises(ValueError, match="matrices"):
        experts.route(x[0], chosen, weight)
    with pytest.raises(ValueError, match="not torch.int32"):
        experts.route(x.int(), chosen, weight)
    with pytest.raises(ValueError, match="matrices"):
        experts.route_gradient(x, chosen[0], weight, x)
    w, y = f(6, 5, 8), f(4, 2, 5)
    with pytest.raises(ValueError, match="device"):
        experts.product(x, w, chosen, y, None)
    with pytest.raises(ValueError, match="wanted"):
        experts.product(x, w[0], chosen, y, None)
    with pytest.raises(ValueError, match="2 slots"):
        experts.product(f(4, 3, 8), w, chosen, y, None)
    with pytest.raises(ValueError, match="device"):
        experts.product_gradient(x, w, chosen, y, x, w, None)
    with pytest.raises(ValueError, match="device"):
        experts.product_workspace_bytes(x, w, chosen)


def test_tensors_handles_are_checked():
    """Rows that a flat buffer cannot have; made and freed without a device (the table's allocation is what fails then)."""
    iwp.load()
    for rows, want in (([(5, 10), (14, 3)], INVALID), ([(-1, 3)], INVALID), ([(0xFFFF0000 - 5, 10)], RANGE), ([], INVALID)):
        with pytest.raises((iwp.IwpError, ValueError)) as e:
            clipping.Tensors(rows)
        assert not isinstance(e.value, iwp.IwpError) or e.value.code == want
    assert iwp._lib.iwp_tensors_create(None, 1, C.byref(C.c_void_p())) == INVALID and iwp._lib.iwp_tensors_create(None, 1, None) == INVALID
    assert iwp._lib.iwp_tensors_workspace_bytes(None, 2) == 0
    assert iwp._hot().iwp_clip(None, [AT], [AT], 1, 1.0, 1.0, AT, AT, 1 << 20, None) == INVALID
