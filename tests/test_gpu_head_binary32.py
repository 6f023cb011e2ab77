"""Binary32 operands of the head are held as two halves relative to their matrix's largest element: 22 bits of an element down to 2^-27 of that,
2^-49 of it below.  One token's hidden states far above the others'."""
import pytest
import torch

from loss_reference import Head, near

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


@pytest.mark.parametrize("power", [20, 30])
def test_a_token_far_above_the_others(gpu_lib, power):
    from paper_1901_01544_amd import losses
    T, D, V = 96, 100, 700
    gen = torch.Generator(device=DEV).manual_seed(power)
    h = torch.randn(T, D, generator=gen, device=DEV)
    w = torch.randn(V, D, generator=gen, device=DEV) * 2.0 / D ** 0.5
    y = torch.randint(V, (T,), generator=gen, device=DEV, dtype=torch.int32)
    h[17] *= 2.0 ** power
    loss, dh, dw = torch.empty(T, device=DEV), torch.empty_like(h), torch.empty_like(w)
    ws = torch.empty(losses.head_workspace_bytes(h, w), dtype=torch.uint8, device=DEV)
    losses.head_cross_entropy(h, w, y, loss, dh, dw, ws)
    ref = Head(h, w, y)
    # what the halves leave of an element, over a logit's sum; a loss has the errors of two logits
    off_z = 2.0 ** -49 * h.double().abs().max() * w.double().abs().sum(1).amax()
    others = torch.arange(T, device=DEV) != 17
    near("loss", loss[others], ref.loss[others], ref.loss_off[others] + 2 * off_z)
