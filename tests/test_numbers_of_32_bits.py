"""Numbers that the C ABI's fields do not hold are turned away, not cut.  No GPU: every call fails its argument checks or has nothing to do."""
import pytest

from paper_1901_01544_amd import clipping, iwp

INVALID, RANGE = iwp.IWP_EINVAL, iwp.IWP_ERANGE
BEYOND = [2 ** 32 + 8, 2 ** 32, -(2 ** 32) + 5, 2 ** 64 + 8, -(2 ** 64) + 8]


@pytest.mark.parametrize("n", BEYOND)
def test_tensors_elements(n):
    with pytest.raises(iwp.IwpError) as e:
        clipping.Tensors([(0, 10), (16, n)])
    assert e.value.code == RANGE


@pytest.mark.parametrize("offset,code", [(2 ** 64 + 16, RANGE), (2 ** 63, RANGE), (-(2 ** 64) + 16, INVALID)])
def test_tensors_offsets(offset, code):
    with pytest.raises(iwp.IwpError) as e:
        clipping.Tensors([(0, 10), (offset, 5)])
    assert e.value.code == code


@pytest.mark.parametrize("n", BEYOND)
def test_plan_rows(n):
    for row, code in (((16, n, 1, 1), RANGE), ((16, 100, n, 1), INVALID), ((16, 100, 1, n + 1), INVALID)):
        with pytest.raises(iwp.IwpError) as e:
            iwp.Plan([(0, 10, 1, 0), row])
        assert e.value.code == code


@pytest.mark.parametrize("name,arguments", [
    ("iwp_route", dict(x=None, ld_x=16, tokens=0, experts=16, dtype=0, bias=None, scores=0, groups=4, top_groups=2, group_top=2, renormalise=0, scale=1.0, keep=None,
                       chosen=None, weight=None, slots=4)),
    ("iwp_route_gradient", dict(x=None, ld_x=16, tokens=0, experts=16, dtype=1, chosen=None, dweight=None, slots=4, scores=0, renormalise=0, scale=1.0, keep=None,
                                plus=None, ld_plus=16, dx=None, ld_dx=16)),
    ("iwp_expert_product", dict(x=None, ld_x=64, by_slot=0, w=0x10000, ld_w=64, step_w=2048, tokens=0, slots=2, experts=4, width=64, out=32, dtype=1, chosen=None,
                                y=None, ld_y=32, ws=None, bytes=0)),
    ("iwp_expert_product_gradient", dict(x=None, ld_x=64, by_slot=0, w=0x10000, ld_w=64, step_w=2048, tokens=0, slots=2, experts=4, width=64, out=32, dtype=1,
                                         chosen=None, dy=None, ld_dy=32, dx=None, ld_dx=64, dw=None, ld_dw=64, step_dw=2048, dw_dtype=0, ws=None, bytes=0))])
def test_hot_calls(name, arguments):
    """As they are the calls have nothing to do; a number that 2^32 or more was added to makes them invalid."""
    iwp.load()
    call = getattr(iwp._hot(), name)
    assert call(*arguments.values(), None) == iwp.IWP_OK
    for what in set(arguments) & {"tokens", "experts", "dtype", "scores", "groups", "top_groups", "group_top", "renormalise", "slots", "by_slot", "width", "out"}:
        for more in (2 ** 32, 2 ** 64, 2 ** 70):
            assert call(*dict(arguments, **{what: arguments[what] + more}).values(), None) == INVALID, (what, more)


def test_workspaces():
    L = iwp.load()
    good = dict(tokens=100, slots=2, experts=8, width=64, out=32, dtype=1, w=0x10000, ld=64, step=2048, by_slot=0, gradient=0)
    assert L.iwp_expert_product_workspace_bytes(*good.values()) > 0
    for what in ("tokens", "slots", "experts", "width", "out", "dtype"):
        assert L.iwp_expert_product_workspace_bytes(*dict(good, **{what: good[what] + 2 ** 32}).values()) == 0, what
