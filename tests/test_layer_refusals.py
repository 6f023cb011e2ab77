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
