"""Groups by the sum of their best two scores, without a bias: inside the chosen groups slots go by the logits, also where scores of 64 bits
are all 1, or all 0."""
import itertools

import pytest
import torch

from loss_reference import near

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
TYPES = [torch.float32, torch.bfloat16, torch.float16]
# experts, groups, top groups, slots: few lanes a token, groups of whole lanes, groups across lanes, more slots than lanes
GROUPS = [(16, 4, 2, 4), (60, 4, 2, 7), (64, 8, 4, 6), (256, 8, 4, 8), (256, 8, 3, 40), (1000, 8, 3, 9), (1024, 8, 5, 12)]


@pytest.fixture(scope="module")
def experts(gpu_lib):
    from paper_1901_01544_amd import experts
    return experts


def logits(T, E, kind, scores):
    """Sigmoid: half of a token's logits, or all, at 40 to 90, where a score of 64 bits is 1 (e^-40 is below 2^-54), the rest between 0.25 and 3.  Softmax: a few of
    0 to 3 and the rest below -800, where it is 0 (e^-760 is below 2^-1074)."""
    gen = torch.Generator(device=DEV).manual_seed(E * 17 + (scores == "softmax"))
    u, few = torch.rand(T, E, generator=gen, device=DEV), torch.rand(T, E, generator=gen, device=DEV)
    if scores == "sigmoid":
        share = torch.where(torch.arange(T, device=DEV) % 3 == 0, 1.0, 0.5)[:, None]
        return torch.where(few < share, 40 + 50 * u, 0.25 + 2.75 * u).to(kind)
    x = torch.where(few < 3.0 / E, 3 * u, -800 - 1200 * u)
    x[:, 0] = 1.0
    return x.to(kind)


@pytest.mark.parametrize("kind", TYPES, ids=str)
@pytest.mark.parametrize("E,groups,top_groups,K", GROUPS)
@pytest.mark.parametrize("scores,renormalise", list(itertools.product(["softmax", "sigmoid"], [False, True])))
def test_slots_by_logits(experts, kind, E, groups, top_groups, K, scores, renormalise):
    T = 203
    x = logits(T, E, kind, scores)
    x[:, E // 2] = float("-inf")
    x[T - 2] = float("-inf")
    x[T - 1] = x[T - 1, 0]
    X = x.double()
    dead = X == float("-inf")
    s = torch.softmax(torch.where(dead.all(1, keepdim=True), 0.0, X), 1) if scores == "softmax" else torch.sigmoid(X)
    s = torch.where(dead, 0.0, s)
    best = torch.where(dead, float("-inf"), s).view(T, groups, -1).sort(dim=2, descending=True).values[:, :, :2]
    total = torch.where(best[:, :, 0] == float("-inf"), float("-inf"), torch.where(best == float("-inf"), 0.0, best).sum(2))
    first = total.sort(dim=1, descending=True, stable=True).indices[:, :top_groups]
    inside = torch.zeros(T, groups, dtype=torch.bool, device=DEV).scatter_(1, first, True).repeat_interleave(E // groups, 1)
    value, at = torch.where(inside, X, float("-inf")).sort(dim=1, descending=True, stable=True)
    there, at = value[:, :K] > float("-inf"), at[:, :K]
    want = torch.where(there, s.gather(1, at), 0.0)
    if renormalise:                                          # shares of what the scores are before any rounding: of logarithms
        log = X if scores == "softmax" else -torch.logaddexp(torch.zeros_like(X), -X)
        log = torch.where(there, log.gather(1, at), float("-inf"))
        want = torch.where(there, torch.softmax(torch.where(there.any(1, keepdim=True), log, 0.0), 1), 0.0)
    chosen = torch.full((T, K), -7, dtype=torch.int32, device=DEV)
    weight = torch.full((T, K), float("nan"), device=DEV)
    experts.route(x, chosen, weight, scores=scores, groups=groups, top_groups=top_groups, group_top=2, renormalise=renormalise)
    assert torch.equal(chosen, torch.where(there, at, -1).to(torch.int32))
    # exponentials of binary32 differences (off by 2^-24 of the difference, then 2^-22), a sum of at most 16 + 6 steps, a quotient
    size = torch.where(dead, 0.0, X.abs()).amax(1, keepdim=True)
    near("weight", weight, want, 2.0 ** -19 * (1 + size) * want)


def test_groups_without_a_choice(experts):
    """A softmax with a logit of +inf has no sums to go by; a sigmoid has."""
    x = torch.arange(64, dtype=torch.float32, device=DEV).repeat(3, 1) / 16
    x[1, 5] = float("inf")
    for scores in ("softmax", "sigmoid"):
        chosen, weight = torch.full((3, 4), -7, dtype=torch.int32, device=DEV), torch.empty(3, 4, device=DEV)
        experts.route(x, chosen, weight, scores=scores, groups=8, top_groups=2, group_top=2)
        assert chosen[0].tolist() == [63, 62, 61, 60] == chosen[2].tolist() and torch.isfinite(weight[[0, 2]]).all()
        if scores == "softmax":
            assert (chosen[1] == -1).all() and weight[1].isnan().all()
        else:
            assert chosen[1].tolist() == [63, 62, 61, 60] and torch.isfinite(weight[1]).all()
