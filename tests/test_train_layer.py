"""The example with a routed layer of matrices and clipped gradients: route, products, losses, clipping and the compression step together.  Without a
GPU: its logic, with the definitions in 64 bits in the kernels' places.  With one: the kernels' gradients against autograd in 64 bits."""
import numpy as np
import pytest
import torch

from layer_reference import Experts, Route, RouteGradient
from paper_1901_01544_amd import clipping, experts, train_lm
from test_train_lm import plain

HOW = dict(width=24, scores="sigmoid")


def plain_layer(monkeypatch):
    def route(x, chosen, weight, scores, renormalise, keep):
        ref = Route(x, chosen.shape[1], scores=scores, renormalise=renormalise, keep=keep)
        chosen.copy_(ref.chosen), weight.copy_(ref.weight)

    def route_gradient(x, chosen, dweight, dx, scores, renormalise, keep):
        dx.copy_(RouteGradient(x, chosen, dweight, scores, renormalise, keep=keep).dx)

    def product(x, w, chosen, y, workspace):
        y.copy_(Experts(x, w, chosen).y)

    def product_gradient(x, w, chosen, dy, dx, dw, workspace):
        ref = Experts(x, w, chosen, dy)
        dx.copy_(ref.dx), dw.copy_(ref.dw)

    class Tensors:
        def __init__(self, rows):
            self.rows = [row[:2] for row in rows]

        def workspace_bytes(self, W):
            return 1

    def clip(tensors, g, out, norm, workspace, max_norm):
        for p, (a, b) in enumerate(zip(g, out)):
            parts = [slice(o, o + n) for o, n in tensors.rows]
            norm[p] = torch.cat([a[s] for s in parts]).double().norm()
            for s in parts:
                b[s] = a[s] * min(1.0, max_norm / norm[p].item())

    for name, f in (("route", route), ("route_gradient", route_gradient), ("product", product), ("product_gradient", product_gradient)):
        monkeypatch.setattr(experts, name, f)
    monkeypatch.setattr(experts, "product_workspace_bytes", lambda *a, **k: 1)
    monkeypatch.setattr(clipping, "Tensors", Tensors)
    monkeypatch.setattr(clipping, "clip", clip)


def worker_gradient(device, taught, seed=0, tokens=200, dim=48, top=8):
    model = train_lm.Model(300, dim, 8, 1 / 8, device, seed, width=HOW["width"])
    worker = train_lm.Worker(model, tokens, dim, top, 2, HOW["scores"], device)
    batch = [x.to(device) for x in train_lm.Text(300, top, seed + 1).batch(tokens)]
    flat = torch.full((model.flat,), 9.0, device=device)
    worker.gradient(batch, model.views(flat), taught)
    return model, worker, batch, flat


def check_gradient(model, worker, batch, flat, taught):
    """Autograd in 64 bits through plain operations, with the experts that were chosen."""
    now, target, index, logit = batch
    w = [x.double().detach().requires_grad_() for x in model.views(model.weights)]
    up, down = (x.unflatten(0, (8, -1)) for x in w[2:4])
    kept = target >= 0
    x = w[0][now]
    logits = x @ w[1].t()
    chosen = logits.detach().topk(2, 1).indices
    s = torch.sigmoid(logits).gather(1, chosen)
    weight = torch.where(kept[:, None], s / s.sum(1, keepdim=True), 0.0)
    inner = torch.nn.functional.silu((up[chosen] @ x[:, None, :, None]).squeeze(3))
    h = x + (weight[:, :, None] * (down[chosen] @ inner[:, :, :, None]).squeeze(3)).sum(1)
    z = h @ w[4].t()
    ce = torch.nn.functional.cross_entropy(z[kept], target[kept].long(), reduction="sum")
    total = ce
    if taught:
        q = torch.log_softmax(logit[kept].double() / 2, 1)
        p = torch.log_softmax(z[kept] / 2, 1).gather(1, index[kept].long())
        total = 0.5 * ce + 0.5 * 4.0 * (q.exp() * (q - p)).sum()
    n = int(kept.sum())
    share = torch.bincount(chosen[kept].reshape(-1), minlength=8).double() / (2 * n)
    soft = torch.softmax(logits, 1)[kept]
    total = total / worker.counted + 0.01 * 8 * (share * soft.mean(0)).sum() + 0.001 * torch.logsumexp(logits[kept], 1).square().mean()
    assert n == worker.counted and int(worker.counts.sum()) == 2 * n
    for got, want in zip(model.views(flat), torch.autograd.grad(total, w)):
        # binary32 throughout, sums over up to 300 terms after each other in the body, the layer and the head
        assert torch.isfinite(got).all()
        assert (got.double() - want).norm() <= 2.0 ** -17 * want.norm() and (got.double() - want).abs().max() <= 2.0 ** -15 * want.abs().max()


def test_logic(monkeypatch):
    plain(monkeypatch)
    plain_layer(monkeypatch)
    for taught in (False, True):
        check_gradient(*worker_gradient("cpu", taught), taught)
    history, counts = train_lm.train(steps=3, device="cpu", clip=0.5, **HOW)
    assert np.isfinite(history).all() and counts.sum() == 2 * 175


@pytest.mark.gpu
@pytest.mark.parametrize("taught", [False, True])
def test_gradients(gpu_lib, taught):
    check_gradient(*worker_gradient("cuda:0", taught), taught)


@pytest.mark.gpu
def test_runs(gpu_lib):
    for how in (HOW, dict(HOW, scores="softmax", clip=0.5), dict(clip=0.5)):
        history, counts = train_lm.train(steps=4, **how)
        assert np.isfinite(history).all() and counts.sum() == 2 * 175 and (counts >= 0).all()


@pytest.mark.gpu
def test_clipped_before_the_step(gpu_lib, monkeypatch):
    """What the step gets has at most the norm that was asked for."""
    from paper_1901_01544_amd import iwp
    seen = []
    step = iwp.step_segmented

    def watched(plan, w, g, *rest, **how):
        seen.append([x.double().norm().item() for x in g])
        return step(plan, w, g, *rest, **how)

    monkeypatch.setattr(iwp, "step_segmented", watched)
    train_lm.train(steps=3, clip=0.25, **HOW)
    assert len(seen) == 3 and all(0 < n <= 0.25 * (1 + 2.0 ** -22) for norms in seen for n in norms) and any(n > 0.2 for norms in seen for n in norms)
