"""The example that runs the losses and the compression step together.  Without a GPU: its logic, with the losses' definitions in 64
bits and the oracle's step in the kernels' places.  With one: the kernels."""
import numpy as np
import pytest
import torch

import oracle
from loss_reference import Balance, Head
from paper_1901_01544_amd import iwp, losses, train_lm


def plain(monkeypatch):
    class Plan:
        def __init__(self, rows):
            self.rows = [tuple(r) for r in rows]

        def step_workspace_bytes(self, W):
            return 1

    def step(plan, w, g, r, leader, eps, scale, idx, val, total, thr, workspace, thr_hint=None):
        w_np, r_np = w.numpy(), [x.numpy() for x in r]
        oracle.step(w_np, [x.numpy() for x in g], r_np, plan.rows, leader.numpy().astype(np.uint32), eps, scale)

    def cross_entropy(h, w, target, loss, dh, dw, workspace, scale=1.0):
        ref = Head(h, w, target, scale=scale)
        loss.copy_(ref.loss), dh.copy_(ref.dh), dw.copy_(ref.dw)

    def distill(h, w, index, logit, loss, dh, dw, workspace, temperature, soft, target, hard, scale):
        ref = Head(h, w, target, index, logit, temperature, hard, soft, scale=scale)
        loss.copy_(ref.loss), dh.copy_(ref.dh), dw.copy_(ref.dw)

    def balance(x, chosen, loss, counts, dx, workspace, balance, z, keep):
        ref = Balance(x, chosen, balance, z, keep)
        loss.copy_(ref.loss), counts.copy_(ref.counts), dx.copy_(ref.dx)

    monkeypatch.setattr(iwp, "Plan", Plan)
    monkeypatch.setattr(iwp, "step_segmented", step)
    monkeypatch.setattr(losses, "head_cross_entropy", cross_entropy)
    monkeypatch.setattr(losses, "head_distill", distill)
    monkeypatch.setattr(losses, "balance", balance)
    monkeypatch.setattr(losses, "head_workspace_bytes", lambda *a, **k: 1)
    monkeypatch.setattr(losses, "balance_workspace_bytes", lambda *a, **k: 1)


def learns(history, counts):
    # what is left is the part of the labels that nothing foretells, so the loss falls to about half
    assert all(np.isfinite(history)) and np.mean(history[-5:]) < 0.75 * history[0], (history[0], history[-5:])
    assert counts.sum() == 2 * (200 - 200 // 8) and (counts >= 0).all()


def test_logic(monkeypatch):
    plain(monkeypatch)
    learns(*train_lm.train(steps=25, device="cpu"))


@pytest.mark.gpu
def test_kernels(gpu_lib):
    learns(*train_lm.train(steps=25))


@pytest.mark.gpu
def test_first_step_matches_the_definitions(gpu_lib, monkeypatch):
    """The same model, tokens and weights: the first losses agree to binary32 sums (over a width of 48, 300 entries, 175 tokens)."""
    here = train_lm.train(steps=1)[0][0]
    with monkeypatch.context() as m:
        plain(m)
        there = train_lm.train(steps=1, device="cpu")[0][0]
    assert abs(here - there) <= 2.0 ** -15 * abs(there)
