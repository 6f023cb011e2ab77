"""Clipping where norms leave binary64 or binary32, where nothing is clipped, and norms without a product."""
import pytest
import torch

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
HALF = 2.0 ** -24
SIZES = pytest.mark.parametrize("n", [3000, 300_000], ids=["one launch", "two"])


@pytest.fixture(scope="module")
def clipping(gpu_lib):
    from paper_1901_01544_amd import clipping
    return clipping


def call(clipping, rows, g, out, **how):
    tensors = clipping.Tensors(rows)
    norm = torch.full((len(g),), float("nan"), device=DEV)
    clipping.clip(tensors, g, out, norm, torch.full((tensors.workspace_bytes(len(g)),), 0xFF, dtype=torch.uint8, device=DEV), **how)
    return norm


@SIZES
@pytest.mark.parametrize("scale", [1e300, -1e300])
def test_norms_beyond_binary64(clipping, n, scale):
    """|scale| times the norm is no number of 64 bits; what is left of the gradient is max_norm long all the same."""
    gen = torch.Generator(device=DEV).manual_seed(n)
    g = 1e12 * torch.randn(n, generator=gen, device=DEV)
    out = torch.empty_like(g)
    norm = call(clipping, [(0, n)], [g], [out], scale=scale, max_norm=5.0)
    want = g.double() * (5.0 / g.double().square().sum().sqrt()) * (1.0 if scale > 0 else -1.0)
    assert norm.item() == float("inf")
    assert ((out.double() - want).abs() <= 1.01 * HALF * want.abs() + 2.0 ** -150).all()


def test_workers_that_32_bits_do_not_hold(clipping):
    tensors = clipping.Tensors([(0, 10)])
    for W in (0, -1, 33, 2 ** 32 + 1):
        with pytest.raises(ValueError):
            tensors.workspace_bytes(W)
