"""The choice of experts and its gradient against their definitions in 64 bits."""
import itertools

import pytest
import torch

from layer_reference import Route, RouteGradient

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
TYPES = [torch.float32, torch.bfloat16, torch.float16]
SIZES = [(1, 1, 1), (1, 8, 2), (5, 3, 3), (200, 8, 2), (67, 60, 4), (1000, 64, 4), (513, 128, 1), (3000, 256, 8), (300, 257, 5), (150, 1000, 16),
         (40, 1024, 1024)]


@pytest.fixture(scope="module")
def experts(gpu_lib):
    from paper_1901_01544_amd import experts
    return experts


def logits(T, E, kind, seed=0):
    gen = torch.Generator(device=DEV).manual_seed(seed * 7919 + T * 31 + E)
    return (2.0 * torch.randn(T, E, generator=gen, device=DEV)).to(kind), gen


def route(experts, x, K, **how):
    T = x.shape[0]
    chosen = torch.full((T, K), -7, dtype=torch.int32, device=DEV)
    weight = torch.full((T, K), float("nan"), device=DEV)
    experts.route(x, chosen, weight, **how)
    return chosen, weight


def gradient(experts, x, chosen, dweight, **how):
    dx = torch.full(x.shape, float("nan"), dtype=x.dtype, device=DEV)
    experts.route_gradient(x, chosen, dweight, dx, **how)
    return dx


@pytest.mark.parametrize("kind", TYPES, ids=str)
@pytest.mark.parametrize("size", SIZES, ids=str)
@pytest.mark.parametrize("scores,renormalise", list(itertools.product(["softmax", "sigmoid"], [False, True])))
def test_route_and_gradient(experts, size, kind, scores, renormalise):
    T, E, K = size
    x, gen = logits(T, E, kind)
    how = dict(scores=scores, renormalise=renormalise, scale=1.5)
    chosen, weight = route(experts, x, K, **how)
    Route(x, K, **how).check(chosen, weight)
    dweight = torch.randn(T, K, generator=gen, device=DEV)
    RouteGradient(x, chosen, dweight, **how).check(gradient(experts, x, chosen, dweight, **how))


@pytest.mark.parametrize("kind", TYPES, ids=str)
@pytest.mark.parametrize("size", SIZES, ids=str)
@pytest.mark.parametrize("scores", ["softmax", "sigmoid"])
def test_bias(experts, size, kind, scores):
    T, E, K = size
    x, gen = logits(T, E, kind, seed=1)
    bias = 0.2 * torch.randn(E, generator=gen, device=DEV)
    Route(x, K, bias, scores, renormalise=True).check(*route(experts, x, K, bias=bias, scores=scores, renormalise=True))


GROUPS = [(16, 2, 1, 4), (16, 16, 3, 3), (60, 4, 2, 7), (256, 8, 4, 8), (256, 8, 7, 40), (96, 3, 1, 1), (1000, 8, 3, 9), (1024, 512, 40, 12), (1024, 1, 1, 5)]


@pytest.mark.parametrize("kind", TYPES, ids=str)
@pytest.mark.parametrize("E,groups,top_groups,K", GROUPS)
@pytest.mark.parametrize("group_top,biased,scores", [(1, False, "softmax"), (2, False, "sigmoid"), (2, True, "sigmoid"), (1, True, "softmax"), (2, False, "softmax")])
def test_groups(experts, kind, E, groups, top_groups, K, group_top, biased, scores):
    if group_top > E // groups:
        pytest.skip("a group of one")
    x, gen = logits(203, E, kind, seed=2)
    x[::5] = torch.where(torch.rand(x[::5].shape, generator=gen, device=DEV) < 0.7, float("-inf"), x[::5].float()).to(kind)
    bias = 0.1 * torch.randn(E, generator=gen, device=DEV) if biased else None
    how = dict(bias=bias, scores=scores, groups=groups, top_groups=top_groups, group_top=group_top, renormalise=True, scale=2.5)
    Route(x, K, **how).check(*route(experts, x, K, **how))


@pytest.mark.parametrize("biased", [False, True])
def test_equal_values_go_to_the_lower_index(experts, biased):
    """Logits of a few values, zeros of both signs among them; the same for groups of equal sums."""
    gen = torch.Generator(device=DEV).manual_seed(5)
    x = torch.randint(-1, 2, (500, 48), generator=gen, device=DEV).float()
    x = torch.where((x == 0) & (torch.rand(x.shape, generator=gen, device=DEV) < 0.5), -0.0, x)
    bias = 0.25 * torch.randint(0, 2, (48,), generator=gen, device=DEV).float() if biased else None
    for how in (dict(), dict(groups=6, top_groups=2), dict(groups=12, top_groups=5, group_top=2)):
        for kind in TYPES:
            Route(x.to(kind), 7, bias, **how).check(*route(experts, x.to(kind), 7, bias=bias, **how))


@pytest.mark.parametrize("scores", ["softmax", "sigmoid"])
def test_scores_next_to_each_other(experts, scores):
    """Biases that make up for the scores' differences up to a few units of binary32's last place: binary64 decides, whatever binary32 says."""
    gen = torch.Generator(device=DEV).manual_seed(6)
    x = torch.randn(1, 64, generator=gen, device=DEV)
    from layer_reference import scores_of
    bias = (0.75 - scores_of(x.double(), scores)[0]).float()
    rows = x.repeat(400, 1)
    moved = torch.randint(0, 64, (400,), generator=gen, device=DEV)
    rows[torch.arange(400, device=DEV), moved] += 2.0 ** -20 * torch.randn(400, generator=gen, device=DEV)
    ref = Route(rows, 12, bias, scores)
    chosen, weight = route(experts, rows, 12, bias=bias, scores=scores)
    ref.check(chosen, weight)
    ref = Route(rows, 12, bias, scores, groups=8, top_groups=3, group_top=2)
    ref.check(*route(experts, rows, 12, bias=bias, scores=scores, groups=8, top_groups=3, group_top=2))


@pytest.mark.parametrize("kind", TYPES, ids=str)
@pytest.mark.parametrize("scores,renormalise", list(itertools.product(["softmax", "sigmoid"], [False, True])))
def test_masks_padding_and_empty_rows(experts, kind, scores, renormalise):
    """Experts masked for a token, fewer of them than slots, none, and padding with NaN in it: forward and back."""
    x, gen = logits(300, 40, kind, seed=3)
    x = torch.where(torch.rand(x.shape, generator=gen, device=DEV) < 0.85, float("-inf"), x.float()).to(kind)
    x[7] = float("-inf")
    x[8] = float("-inf")
    x[8, 33] = -60.0
    keep = (torch.rand(300, generator=gen, device=DEV) > 0.3).to(torch.uint8)
    keep[6:9] = 255
    how = dict(scores=scores, renormalise=renormalise)
    ref = Route(x, 6, keep=keep, **how)
    dweight = torch.randn(300, 6, generator=gen, device=DEV)
    back = RouteGradient(x, ref.chosen, dweight, keep=keep, **how)
    x[keep == 0] = float("nan")
    dweight[ref.chosen < 0] = float("nan")
    for bias in (None, torch.zeros(40, device=DEV)):
        chosen, weight = route(experts, x, 6, keep=keep, bias=bias, **how)
        ref.check(chosen, weight)
    assert (chosen[7] == -1).all() and chosen[8, 0] == 33 and (chosen[keep == 0] == -1).all()
    dx = gradient(experts, x, chosen, dweight, keep=keep, **how)
    back.check(dx)
    assert (dx[keep == 0] == 0).all() and (dx[7] == 0).all()


def test_nan_and_infinity(experts):
    x, _ = logits(6, 12, torch.float32, seed=4)
    x[0, 3] = float("nan")
    x[1] = float("nan")
    x[2, 5] = float("inf")
    for scores, renormalise, bias in itertools.product(["softmax", "sigmoid"], [False, True], [None, torch.zeros(12, device=DEV)]):
        chosen, weight = route(experts, x, 4, scores=scores, renormalise=renormalise, bias=bias)
        assert weight[:2].isnan().all() and (chosen[1] == -1).all() and 3 not in chosen[0].tolist() and len(set(chosen[0].tolist())) == 4
        assert torch.isfinite(weight[3:]).all()
        if scores == "sigmoid":
            assert torch.isfinite(weight[2]).all() and chosen[2, 0] == 5
        else:
            assert weight[2].isnan().all()
    bias = torch.zeros(12, device=DEV)
    bias[2], bias[4], bias[9] = float("nan"), float("-inf"), float("inf")
    chosen, weight = route(experts, x[3:], 10, bias=bias)
    assert (chosen[:, 0] == 9).all() and not ((chosen == 2) | (chosen == 4)).any() and torch.isfinite(weight).all()


@pytest.mark.parametrize("scores", ["softmax", "sigmoid"])
def test_small_scores_renormalised(experts, scores):
    """Scores far below binary32's range still have shares."""
    x, gen = logits(50, 16, torch.float32, seed=7)
    x = x - 300.0 - 40.0 * torch.arange(50, device=DEV)[:, None]
    how = dict(scores=scores, renormalise=True)
    chosen, weight = route(experts, x, 4, **how)
    shifted = Route(x + 300.0 + 40.0 * torch.arange(50, device=DEV)[:, None], 4, renormalise=True)      # a sigmoid is an exponential there
    exact = Route(x, 4, renormalise=True)
    assert torch.equal(chosen, exact.chosen) and torch.equal(chosen, shifted.chosen)
    assert ((weight.double().sum(1) - 1).abs() < 2.0 ** -20).all()
    assert ((weight.double() - exact.weight).abs() <= exact.off + 2.0 ** -24).all()
    dweight = torch.randn(50, 4, generator=gen, device=DEV)
    RouteGradient(x, chosen, dweight, renormalise=True).check(gradient(experts, x, chosen, dweight, **how))


@pytest.mark.parametrize("kind", TYPES, ids=str)
@pytest.mark.parametrize("shift", [0, 1, 4])
@pytest.mark.parametrize("scores", ["softmax", "sigmoid"])
def test_strided_rows_and_plus(experts, kind, shift, scores):
    for E in (12, 64, 256):
        x0, gen = logits(130, E, kind, seed=8)
        x = torch.full((130, E + 11), float("nan"), dtype=kind, device=DEV)[:, shift:shift + E]
        x.copy_(x0)
        chosen, weight = route(experts, x, 3, scores=scores)
        Route(x0, 3, scores=scores).check(chosen, weight)
        dweight = torch.randn(130, 3, generator=gen, device=DEV)
        plus = torch.randn(130, E, generator=gen, device=DEV).to(kind)
        keep = (torch.arange(130, device=DEV) % 4 != 0).to(torch.uint8)
        ref = RouteGradient(x0, chosen, dweight, scores=scores, keep=keep, plus=plus)
        whole = torch.full((130, E + 7), 9.0, dtype=kind, device=DEV)
        dx = whole[:, shift:shift + E]
        experts.route_gradient(x, chosen, dweight, dx, scores=scores, keep=keep, plus=plus)
        ref.check(dx)
        assert torch.equal(dx[keep == 0], plus[keep == 0])
        assert (whole[:, :shift] == 9).all() and (whole[:, shift + E:] == 9).all()
        dx.copy_(plus)                                                  # onto itself
        experts.route_gradient(x, chosen, dweight, dx, scores=scores, keep=keep, plus=dx)
        ref.check(dx)


def test_an_expert_twice_and_slots_of_nobody(experts):
    x, gen = logits(90, 20, torch.float32, seed=9)
    chosen = torch.randint(-2, 23, (90, 9), generator=gen, device=DEV, dtype=torch.int32)
    dweight = torch.randn(90, 9, generator=gen, device=DEV)
    for scores, renormalise in itertools.product(["softmax", "sigmoid"], [False, True]):
        how = dict(scores=scores, renormalise=renormalise)
        RouteGradient(x, chosen, dweight, **how).check(gradient(experts, x, chosen, dweight, **how))


def test_no_tokens(experts):
    x = torch.empty(0, 16, device=DEV)
    chosen, weight = route(experts, x, 2)
    assert gradient(experts, x, chosen, weight).shape == (0, 16)


@pytest.mark.parametrize("scores,renormalise", list(itertools.product(["softmax", "sigmoid"], [False, True])))
def test_gradient_against_differences(experts, scores, renormalise):
    """Logits at least 0.25 apart, so a step of 2^-6 changes no choice.  Along a unit direction a weight's third derivative is below 4, a
    difference of binary32 weights (below 1, off by 2^-19 (1 + 8) each, weighted by dweight) is divided by twice the step."""
    gen = torch.Generator(device=DEV).manual_seed(10)
    T, E, K = 30, 24, 5
    x = 0.25 * torch.rand(T, E, generator=gen, device=DEV).argsort(1).float() - 3.0
    dweight = torch.randn(T, K, generator=gen, device=DEV)
    v = torch.randn(T, E, generator=gen, device=DEV)
    v = v / v.norm(dim=1, keepdim=True)
    how = dict(scores=scores, renormalise=renormalise)
    chosen, _ = route(experts, x, K, **how)
    step = 2.0 ** -6
    value = []
    for to in (step, -step):
        c, w = route(experts, x + to * v, K, **how)
        assert torch.equal(c, chosen)
        value.append((w.double() * dweight).sum(1))
    slope = (gradient(experts, x, chosen, dweight, **how).double() * v).sum(1)
    most = dweight.double().abs().sum(1)
    assert ((value[0] - value[1]) / (2 * step) - slope).abs().le(most * (4 * step ** 2 / 6 + 9 * 2.0 ** -19 / step)).all()


@pytest.mark.parametrize("size", [(60, 8, 2), (5000, 64, 4), (20000, 256, 8)], ids=str)
def test_same_bytes_on_another_stream_and_in_a_graph(experts, size):
    T, E, K = size
    x, gen = logits(T, E, torch.bfloat16, seed=11)
    bias = 0.1 * torch.randn(E, generator=gen, device=DEV)
    dweight = torch.randn(T, K, generator=gen, device=DEV)
    how = dict(scores="sigmoid", renormalise=True)

    def both(chosen, weight, dx):
        experts.route(x, chosen, weight, bias=bias, groups=4, top_groups=2, group_top=2, **how)
        experts.route_gradient(x, chosen, dweight, dx, **how)
        return chosen, weight, dx

    def empty():
        return torch.empty(T, K, dtype=torch.int32, device=DEV), torch.empty(T, K, device=DEV), torch.empty_like(x)

    first = both(*empty())
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        second = both(*empty())
    torch.cuda.synchronize()
    third = empty()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        both(*third)
    for _ in range(3):
        for t in third:
            t.fill_(5)
        graph.replay()
        torch.cuda.synchronize()
        for a, b, c in zip(first, second, third):
            assert torch.equal(a, b) and torch.equal(a, c)


@pytest.mark.parametrize("kind", TYPES, ids=str)
@pytest.mark.parametrize("E", [8, 100, 256, 1024])
def test_all_alike_and_masked_by_the_lowest_value(experts, kind, E):
    """More equal logits than a token's candidates have room for; masks of the type's lowest value instead of -inf, for some and for all."""
    x = torch.zeros(70, E, dtype=kind, device=DEV)
    gen = torch.Generator(device=DEV).manual_seed(12)
    lowest = torch.finfo(kind).min
    x[20:] = torch.randn(50, E, generator=gen, device=DEV).to(kind)
    x[20:40, E // 4:] = lowest
    x[40:60, 3:] = lowest
    x[60:] = lowest
    x[65:, E // 2] = torch.finfo(kind).max
    K = 4
    for how in (dict(), dict(renormalise=True), dict(scores="sigmoid"), dict(bias=torch.zeros(E, device=DEV)),
                dict(bias=torch.zeros(E, device=DEV), scores="sigmoid", groups=4, top_groups=2, group_top=2)):
        chosen, weight = route(experts, x, K, **how)
        ref = Route(x, K, **how)
        assert torch.equal(chosen, ref.chosen)
        assert (chosen[:20] == torch.arange(K, device=DEV)).all()
        # differences to the lowest value round to it, and its exponential is 0 either way: the bound of the values that are ordinary ones
        small = 2.0 ** -19 * 8 * ref.weight.abs() + 2.0 ** -140
        assert ((weight.double() - ref.weight).abs() <= small).all()
        dx = gradient(experts, x, chosen, torch.ones(70, K, device=DEV), **{k: v for k, v in how.items() if k in ("scores", "renormalise")})
        assert torch.isfinite(dx).all()


def test_rows_beyond_32_bits(experts):
    """2^20 tokens, rows 16 KB apart: checked at both ends."""
    T, E = 1 << 20, 48
    x = torch.empty(T * 8192, dtype=torch.bfloat16, device=DEV).view(T, 8192)[:, 100:100 + E]
    x0, gen = logits(T, E, torch.bfloat16, seed=13)
    x.copy_(x0)
    dweight = torch.randn(T, 3, generator=gen, device=DEV)
    bias = 0.1 * torch.randn(E, generator=gen, device=DEV)
    chosen, weight = route(experts, x, 3, bias=bias)
    experts.route_gradient(x, chosen, dweight, x, plus=x)
    for part in (slice(0, 100), slice(T - 100, T)):
        Route(x0[part], 3, bias).check(chosen[part], weight[part])
        RouteGradient(x0[part], chosen[part], dweight[part], plus=x0[part]).check(x[part].contiguous())
