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
