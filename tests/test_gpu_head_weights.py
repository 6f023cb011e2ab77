"""Weights of the head's tokens far apart, infinite or not a number: what a token's gradient row does not depend on must not change it,
and a small weight must not cost its row any bits.

The bounds of a gradient row come from the definition's with every weight 1: the row is that one's times its weight, and so is all
that it may be off by.  Those of the weight's gradient are summed here: each token's share is off by the rounding of its dz and by
its logits' error, both in proportion to its own coefficient, and, where operands are kept in parts or in fp16, by what the scaling
of its hidden states to the largest coefficient leaves of them."""
import pytest
import torch

from loss_reference import UNIT, Head, near

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
TYPES = [torch.float32, torch.bfloat16, torch.float16]
INF, NAN = float("inf"), float("nan")


@pytest.fixture(scope="module")
def losses(gpu_lib):
    from paper_1901_01544_amd import losses
    return losses


def inputs(T, D, V, kind, seed):
    gen = torch.Generator(device=DEV).manual_seed(seed)
    h = torch.randn(T, D, generator=gen, device=DEV).to(kind)
    w = (torch.randn(V, D, generator=gen, device=DEV) * 3.0 / D ** 0.5).to(kind)
    y = torch.randint(V, (T,), generator=gen, device=DEV, dtype=torch.int32)
    index = torch.stack([torch.randperm(V, generator=gen, device=DEV)[:9] for _ in range(T)]).to(torch.int32)
    logit = 3.0 * torch.randn(T, 9, generator=gen, device=DEV)
    return h, w, y, index, logit, gen


def call(losses, h, w, y, weight, scale, piece, teacher=None, dw_dtype=None, mix=(0.4, 0.6, 2.0)):
    loss = torch.full((h.shape[0],), NAN, device=DEV)
    dh = torch.full_like(h, NAN)
    dw = torch.full(w.shape, NAN, dtype=dw_dtype or w.dtype, device=DEV)
    top = teacher[0].shape[1] if teacher else 0
    ws = torch.full((losses.head_workspace_bytes(h, w, top=top, piece=piece),), 0xFF, dtype=torch.uint8, device=DEV)
    if teacher:
        hard, soft, t = mix
        losses.head_distill(h, w, *teacher, loss, dh, dw, ws, temperature=t, soft=soft, target=y, hard=hard, weight=weight, scale=scale,
                            piece=piece)
    else:
        losses.head_cross_entropy(h, w, y, loss, dh, dw, ws, weight=weight, scale=scale, piece=piece)
    return loss, dh, dw


@pytest.mark.parametrize("kind", TYPES, ids=str)
@pytest.mark.parametrize("bad,distill", [(INF, False), (-INF, False), (NAN, False), (INF, True), (-INF, True), (NAN, True), (3e38, True)], ids=str)
@pytest.mark.parametrize("piece", [0, 256])
def test_a_weight_without_bounds_stays_with_its_token(losses, kind, bad, distill, piece):
    """Losses and gradient rows of the other tokens to the last bit as with a weight of 1 there.  3e38: a finite weight, whose coefficient is
    not (the label's part is taken eight times)."""
    T, D, V = 150, 72, 700
    h, w, y, index, logit, gen = inputs(T, D, V, kind, 1)
    teacher = (index, logit) if distill else None
    at = 70
    weight = 0.5 + torch.rand(T, generator=gen, device=DEV)
    weight[at] = 1.0
    others = torch.arange(T, device=DEV) != at
    args = dict(scale=0.25, piece=piece, teacher=teacher, mix=(8.0, 0.6, 2.0))
    loss, dh, _ = call(losses, h, w, y, weight, **args)
    assert loss.isfinite().all() and dh.isfinite().all()
    weight[at] = bad
    loss2, dh2, dw2 = call(losses, h, w, y, weight, **args)
    assert torch.equal(loss2[others], loss[others])
    assert torch.equal(dh2[others], dh[others])
    assert not loss2[at].isfinite() and not dh2[at].isfinite().any() and not dw2.isfinite().any()


@pytest.mark.parametrize("kind", TYPES, ids=str)
def test_every_weight_without_bounds(losses, kind):
    h, w, y, _, _, _ = inputs(40, 64, 300, kind, 2)
    y[::2] = -1
    loss, dh, dw = call(losses, h, w, y, torch.full((40,), INF, device=DEV), 1.0, 0)
    assert (loss[::2] == 0).all() and (dh[::2] == 0).all()
    assert not loss[1::2].isfinite().any() and not dh[1::2].isfinite().any() and not dw.isfinite().any()


# binary32 and bf16 have the range for any spread; what fp16 holds of a gradient ends at 2^-24, whatever it is computed from
SPREADS = [(torch.float32, 20), (torch.float32, 60), (torch.bfloat16, 60), (torch.float16, 9)]


@pytest.mark.parametrize("kind,spread", SPREADS, ids=str)
@pytest.mark.parametrize("distill", [False, True])
@pytest.mark.parametrize("piece", [0, 256])
def test_gradient_rows_of_small_weights(losses, kind, spread, distill, piece):
    """Weights from 1 down to 2^-spread: each row as exact as if all weights were its own."""
    T, D, V = 130, 64, 700
    h, w, y, index, logit, gen = inputs(T, D, V, kind, 3)
    weight = torch.exp2(-spread * torch.rand(T, generator=gen, device=DEV))
    weight[::7] *= -1.0
    scale = 2.0 ** 9 if kind == torch.float16 else 1.0
    teacher = (index, logit) if distill else None
    _, dh, _ = call(losses, h, w, y, weight, scale, piece, teacher)
    ref = Head(h, w, y, index, logit, 2.0, 0.4, 0.6, scale=scale) if distill else Head(h, w, y, scale=scale)
    a = weight.double()[:, None]
    near("dh", dh, ref.dh * a, ref.dh_off * a.abs())


def weight_gradient(h, w, y, weight, scale):
    """dW of the cross entropy and what it may be off by."""
    kind = h.dtype
    H, W, a = h.double(), w.double(), weight.double()[:, None] * scale
    z = H @ W.t()
    p = torch.softmax(z, 1)
    one = torch.zeros_like(z).scatter_(1, y.long()[:, None], 1.0)
    dz, grown = a * (p - one), a.abs() * (p + one)
    off_z = 2.0 ** -20 * (H.norm(dim=1, keepdim=True) * W.norm(dim=1)).amax(1, keepdim=True)
    off = grown * (2 * off_z + 2.0 ** -19 * (1 + z.abs()))
    if kind != torch.float32:
        off = off + UNIT[kind] * dz.abs()
    if kind == torch.bfloat16:                              # kept as distances to the largest logit of 128 entries at most, in 16 bits
        off = off + 2.0 ** -11 * grown * (z.amax(1, keepdim=True) - z)
    # dz itself: relative to the token's coefficient, to twice that for its power of two
    off = off + a.abs() * {torch.float32: 2.0 ** -48, torch.bfloat16: 0.0, torch.float16: 2.0 ** -38}[kind]
    dw_off = off.t() @ H.abs() + 2.0 ** -20 * (dz.abs().t() @ H.abs())
    # hidden states times a power of two for the token's coefficient: halves end at 2^-36 where the largest is 2^13 to 2^14, fp16 at 2^-25,
    # and a dz is relative to a power of two that is up to half its coefficient: 2 2^-49 and 2 2^-38 of the largest
    ends = {torch.float32: 2.0 ** -48, torch.bfloat16: 0.0, torch.float16: 2.0 ** -37}[kind]
    relative = (dz / a).abs().t() @ (H != 0).double()
    return dz.t() @ H, dw_off + ends * relative * a.abs().max() * H.abs().max()


@pytest.mark.parametrize("kind,spread", SPREADS[:3] + [(torch.float32, 30), (torch.float16, 20)], ids=str)
@pytest.mark.parametrize("dw_dtype", [None, torch.float32], ids=str)
@pytest.mark.parametrize("piece", [0, 256])
def test_weight_gradient_of_small_weights(losses, kind, spread, dw_dtype, piece):
    """Two tokens that nothing ties: the second's entries are the only ones in their half of the width, and of a weight of 2^-spread."""
    T, D, V = 64, 64, 600
    h, w, y, _, _, gen = inputs(T, D, V, kind, 4)
    first = torch.arange(T, device=DEV) % 2 == 0
    h[first, D // 2:] = 0.0
    h[~first, :D // 2] = 0.0
    weight = torch.where(first, 1.0, 2.0 ** -spread).float() * (0.75 + torch.rand(T, generator=gen, device=DEV))
    scale = 2.0 ** 6 if kind == torch.float16 else 1.0
    _, _, dw = call(losses, h, w, y, weight, scale, piece, dw_dtype=dw_dtype)
    want, off = weight_gradient(h, w, y, weight, scale)
    near("dw", dw, want, off)


@pytest.mark.parametrize("kind", TYPES, ids=str)
def test_same_bytes_for_weights_of_one_size(losses, kind):
    """Weights that share a power of two take hidden states as they are, others a copy: a token of no effect must not change a byte of dW."""
    T, D, V = 100, 64, 500
    h, w, y, _, _, gen = inputs(T, D, V, kind, 5)
    weight = 1.0 + torch.rand(T, generator=gen, device=DEV) * 0.99
    h[50] = 0.0
    _, _, dw = call(losses, h, w, y, weight, 1.0, 0)
    weight[50] = 2.0 ** -6                                   # its row of zeros adds nothing, whatever its weight
    _, _, dw2 = call(losses, h, w, y, weight, 1.0, 0)
    assert torch.equal(dw, dw2)
