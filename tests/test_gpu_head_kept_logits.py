"""What a bf16 head's gradient loses by the logits that are kept from one pass to the next, entry by entry.

The hidden state is a unit vector and the weight's first column holds the logits, exact in bf16, so a row of dW is an entry of dz as it
was stored.  With u = 2^-8 (bf16) an entry p of a softmax may be off by u p for its rounding, by 2^-19 (1 + |z|) p for binary32
exponentials, and, where its logit was kept, by what 2^-13 (1 + d) moves the exponential, d its distance to the largest of
its group: 128 neighbouring entries at most, from a multiple of that on."""
import pytest
import torch

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
# tokens and vocabulary: every kind of tile
SIZES = [(1, 1000), (128, 20480), (256, 40960)]


@pytest.fixture(scope="module")
def losses(gpu_lib):
    from paper_1901_01544_amd import losses
    return losses


def head(T, V, reach, seed):
    gen = torch.Generator(device=DEV).manual_seed(seed)
    z = (-reach * torch.rand(V, generator=gen, device=DEV)).to(torch.bfloat16)
    w = torch.zeros(V, 8, dtype=torch.bfloat16, device=DEV)
    w[:, 0] = z
    h = torch.zeros(T, 8, dtype=torch.bfloat16, device=DEV)
    h[:, 0] = 1.0
    y = torch.full((T,), -1, dtype=torch.int32, device=DEV)
    y[T - 1] = 3                                            # one token counts: dW is its dz
    z = z.double()
    groups = torch.nn.functional.pad(z, (0, -V % 128), value=float("-inf")).view(-1, 128).amax(1)
    return h, w, y, z, groups.repeat_interleave(128)[:V] - z


def run(losses, h, w, piece, f, top=0):
    loss, dh, dw = torch.empty(h.shape[0], device=DEV), torch.empty_like(h), torch.empty(w.shape, device=DEV)
    ws = torch.full((losses.head_workspace_bytes(h, w, top=top, piece=piece),), 0xFF, dtype=torch.uint8, device=DEV)
    f(loss, dh, dw, ws)
    return dw[:, 0].double()


def check(got, p, z, d, kept, t):
    """p: the entries, from logits z / t."""
    off = 2.0 ** -8 + 2.0 ** -19 * (1 + z.abs() / t) + torch.where(kept, torch.expm1(2.0 ** -13 * (1 + d) / t), 0.0)
    over = ((got - p).abs() / p / off)
    assert over.max() <= 1.0, "entry %d: %.3g of what is allowed, distance %.3g" % (over.argmax(), over.max(), d[over.argmax()])


@pytest.mark.parametrize("size", SIZES, ids=str)
@pytest.mark.parametrize("reach", [4.0, 60.0])
@pytest.mark.parametrize("pieces", [1, 3])
def test_cross_entropy(losses, size, reach, pieces):
    T, V = size
    h, w, y, z, d = head(T, V, reach, 1)
    piece = 0 if pieces == 1 else (V + 2) // 3
    got = run(losses, h, w, piece, lambda loss, dh, dw, ws: losses.head_cross_entropy(h, w, y, loss, dh, dw, ws, piece=piece))
    last = 0 if pieces == 1 else (V - 1) // ((piece + 255) // 256 * 256) * ((piece + 255) // 256 * 256)
    entry = torch.arange(V, device=DEV)
    others = entry != 3
    check(got[others], torch.softmax(z, 0)[others], z[others], d[others], (entry >= last)[others], 1.0)


@pytest.mark.parametrize("size", SIZES, ids=str)
@pytest.mark.parametrize("reach,t", [(45.0, 0.75), (250.0, 8.0), (50000.0, 1000.0)], ids=str)
def test_distill(losses, size, reach, t):
    """Soft gradient alone; at high temperatures far entries count."""
    T, V = size
    h, w, y, z, d = head(T, V, reach, 2)
    index = y.clone()[:, None].contiguous()                 # the one token's only entry
    logit = torch.zeros(T, 1, device=DEV)
    got = run(losses, h, w, 0, lambda loss, dh, dw, ws: losses.head_distill(h, w, index, logit, loss, dh, dw, ws, temperature=t, scale=1.0 / t), 1)
    others = torch.arange(V, device=DEV) != 3
    p = torch.softmax(z / t, 0)[others]
    check(got[others], p, z[others], d[others], torch.ones_like(others)[others], t)
