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


@SIZES
@pytest.mark.parametrize("onto", [False, True], ids=["apart", "in place"])
def test_infinity_and_nan_without_a_largest_norm(clipping, n, onto):
    """max_norm = inf scales alone: an infinity stays one, the rest is scaled, the norm tells.  A NaN makes all of it NaN."""
    for scale in (1.0, -0.25):
        g = [torch.full((n,), 3.0, device=DEV) for _ in range(3)]
        g[0][n // 2], g[1][n - 1] = float("inf"), float("nan")
        out = g if onto else [torch.empty_like(x) for x in g]
        norm = call(clipping, [(0, n)], g, out, scale=scale)
        assert norm[0].item() == float("inf") and norm[1].isnan()
        want = torch.full((n,), 3.0 * scale, device=DEV)
        assert torch.equal(out[2], want)
        want[n // 2] = float("inf") * scale
        assert torch.equal(out[0], want)
        assert out[1].isnan().all()


def test_norms_alone_of_workers_beyond_the_cache(clipping):
    """Norms alone take a grid of their own; every worker's against its own, the quiet one's too."""
    rows = [(0, 20_000_001), (20_000_100, 25_000_003)]
    gen = torch.Generator(device=DEV).manual_seed(5)
    g = [size * torch.randn(45_000_103, generator=gen, device=DEV) for size in (1.0, 2.0, 4e-3)]
    norm = call(clipping, rows, g, None, max_norm=100.0)
    for p, x in enumerate(g):
        want = sum(x[o:o + n].double().square().sum() for o, n in rows).sqrt()
        assert abs(norm[p].double() - want) <= 1.01 * HALF * want, p


def test_workers_that_32_bits_do_not_hold(clipping):
    tensors = clipping.Tensors([(0, 10)])
    for W in (0, -1, 33, 2 ** 32 + 1):
        with pytest.raises(ValueError):
            tensors.workspace_bytes(W)
