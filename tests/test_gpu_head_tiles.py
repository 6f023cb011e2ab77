"""The head's losses at sizes that take every kind of tile, more tokens than one round of their numbering, and teachers with many entries
in one place."""
import pytest
import torch

from loss_reference import Head

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
TYPES = [torch.float32, torch.bfloat16, torch.float16]


@pytest.fixture(scope="module")
def losses(gpu_lib):
    from paper_1901_01544_amd import losses
    return losses


def run(losses, T, D, V, kind, top=0, piece=0, near=0):
    gen = torch.Generator(device=DEV).manual_seed(T + 3 * D + 7 * V + top)
    h = torch.randn(T, D, generator=gen, device=DEV).to(kind)
    w = (torch.randn(V, D, generator=gen, device=DEV) * 2.0 / D ** 0.5).to(kind)
    y = torch.randint(V, (T,), generator=gen, device=DEV, dtype=torch.int32)
    y[torch.rand(T, generator=gen, device=DEV) < 0.3] = -1
    weight = torch.rand(T, generator=gen, device=DEV) + 0.5
    loss, dh, dw = torch.empty(T, device=DEV), torch.full_like(h, float("nan")), torch.full_like(w, float("nan"))
    ws = torch.full((losses.head_workspace_bytes(h, w, top=top, piece=piece),), 0xFF, dtype=torch.uint8, device=DEV)
    if top:
        first = torch.randint(max(1, near or V - top), (T, 1), generator=gen, device=DEV)
        index = ((first + torch.arange(top, device=DEV)) % V).to(torch.int32)      # neighbours: many in one tile
        logit = 2.0 * torch.randn(T, top, generator=gen, device=DEV)
        losses.head_distill(h, w, index, logit, loss, dh, dw, ws, temperature=2.0, soft=0.7, target=y, hard=0.3, weight=weight, piece=piece)
        Head(h, w, y, index, logit, 2.0, 0.3, 0.7, weight=weight).check(loss, dh, dw)
    else:
        losses.head_cross_entropy(h, w, y, loss, dh, dw, ws, weight=weight, piece=piece)
        Head(h, w, y, weight=weight).check(loss, dh, dw)


@pytest.mark.parametrize("kind", TYPES, ids=str)
@pytest.mark.parametrize("size", [(300, 72, 20011), (300, 72, 41000), (50, 72, 30000), (2500, 40, 500), (1100, 200, 9000)], ids=str)
def test_tiles(losses, size, kind):
    run(losses, *size, kind)


@pytest.mark.parametrize("kind", TYPES, ids=str)
@pytest.mark.parametrize("size,piece", [((300, 72, 20011), 10240), ((40, 64, 5000), 1024), ((300, 72, 41000), 20480)], ids=str)
def test_tiles_in_pieces(losses, size, piece, kind):
    run(losses, *size, kind, piece=piece)


@pytest.mark.parametrize("kind", TYPES, ids=str)
@pytest.mark.parametrize("size,top,near", [((300, 72, 20011), 20, 0), ((300, 72, 41000), 70, 0), ((130, 64, 3000), 200, 10), ((50, 40, 2000), 33, 5)],
                         ids=str)
@pytest.mark.parametrize("piece", [0, 1536])
def test_teachers_entries_close_together(losses, size, top, near, piece, kind):
    run(losses, *size, kind, top=top, near=near, piece=piece)
