"""Cross entropy and distillation through the head against their definitions in 64 bits: types, odd sizes, pieces of the vocabulary,
tokens that do not count, strides, and what stands in places that nothing may be read from."""
import pytest
import torch

from loss_reference import Head

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
TYPES = [torch.float32, torch.bfloat16, torch.float16]
SIZES = [(1, 1, 1), (1, 8, 2), (2, 3, 5), (3, 64, 1000), (64, 40, 257), (70, 130, 300), (129, 72, 513), (257, 200, 1030), (300, 264, 2000)]


def inputs(T, D, V, kind, seed=0, spread=1.0):
    gen = torch.Generator(device=DEV).manual_seed(seed * 1000 + T * 31 + D * 7 + V)
    h = torch.randn(T, D, generator=gen, device=DEV)
    w = torch.randn(V, D, generator=gen, device=DEV) * (3.0 * spread / D ** 0.5)
    y = torch.randint(V, (T,), generator=gen, device=DEV, dtype=torch.int32)
    return h.to(kind), w.to(kind), y, gen


def outputs(h, w, dw_dtype=None):
    nan = float("nan")
    return (torch.full((h.shape[0],), nan, device=DEV), torch.full_like(h, nan),
            torch.full(w.shape, nan, dtype=dw_dtype or w.dtype, device=DEV))


def workspace(losses, h, w, top=0, piece=0):
    # whatever a workspace holds must not matter: NaN patterns in binary32 and fp16
    return torch.full((losses.head_workspace_bytes(h, w, top=top, piece=piece),), 0xFF, dtype=torch.uint8, device=DEV)


@pytest.fixture(scope="module")
def losses(gpu_lib):
    from paper_1901_01544_amd import losses
    return losses


@pytest.mark.parametrize("kind", TYPES, ids=str)
@pytest.mark.parametrize("size", SIZES, ids=str)
def test_cross_entropy(losses, size, kind):
    T, D, V = size
    h, w, y, _ = inputs(T, D, V, kind)
    loss, dh, dw = outputs(h, w)
    losses.head_cross_entropy(h, w, y, loss, dh, dw, workspace(losses, h, w), scale=1.0 / T)
    Head(h, w, y, scale=1.0 / T).check(loss, dh, dw)


@pytest.mark.parametrize("kind", TYPES, ids=str)
@pytest.mark.parametrize("piece", [1, 256, 700, 1792, 5000])
def test_pieces(losses, piece, kind):
    h, w, y, _ = inputs(140, 96, 1793, kind, seed=1)
    loss, dh, dw = outputs(h, w)
    losses.head_cross_entropy(h, w, y, loss, dh, dw, workspace(losses, h, w, piece=piece), piece=piece)
    Head(h, w, y).check(loss, dh, dw)


@pytest.mark.parametrize("kind", TYPES, ids=str)
@pytest.mark.parametrize("piece", [0, 256])
def test_tokens_that_do_not_count(losses, kind, piece):
    """Labels outside the vocabulary, weights of zero and below; rows of NaN and infinities where nothing counts."""
    T, D, V = 333, 80, 600
    h, w, y, gen = inputs(T, D, V, kind, seed=2)
    weight = torch.rand(T, generator=gen, device=DEV) * 2 - 0.5
    y[::3] = -100
    y[1] = V
    y[2] = 2 ** 31 - 1
    weight[4:20] = 0.0
    clean = h.clone()
    out = (y < 0) | (y >= V) | (weight == 0)
    h[out] = float("nan")
    h[4] = float("inf")
    weight[0] = float("nan")            # of a token whose label already keeps it out
    assert out[0] and out[4]
    loss, dh, dw = outputs(h, w)
    losses.head_cross_entropy(h, w, y, loss, dh, dw, workspace(losses, h, w, piece=piece), weight=weight, scale=0.25, piece=piece)
    Head(clean, w, y, weight=torch.where(out, 0.0, weight), scale=0.25).check(loss, dh, dw)


@pytest.mark.parametrize("kind", TYPES, ids=str)
def test_nothing_counts(losses, kind):
    h, w, y, _ = inputs(65, 64, 300, kind)
    loss, dh, dw = outputs(h, w)
    losses.head_cross_entropy(h, w, torch.full_like(y, -1), loss, dh, dw, workspace(losses, h, w))
    assert (loss == 0).all() and (dh == 0).all() and (dw == 0).all()
    loss, dh, dw = outputs(h[:0], w)
    losses.head_cross_entropy(h[:0], w, y[:0], loss, dh, dw, workspace(losses, h[:0], w))
    assert (dw == 0).all()


@pytest.mark.parametrize("kind", TYPES, ids=str)
@pytest.mark.parametrize("shift", [0, 1, 8])
def test_strided_rows(losses, kind, shift):
    """Operands and gradients as parts of wider buffers, at even and odd places; nothing beside them is read or written."""
    T, D, V = 90, 120, 410
    h0, w0, y, _ = inputs(T, D, V, kind, seed=3)

    def within(rows, columns, dtype, fill):
        whole = torch.full((rows, columns + 40), fill, dtype=dtype, device=DEV)
        return whole, whole[:, shift:shift + columns]

    _, h = within(T, D, kind, float("nan"))
    _, w = within(V, D, kind, float("nan"))
    h.copy_(h0)
    w.copy_(w0)
    dh_all, dh = within(T, D, kind, 7.0)
    for dw_kind in {kind, torch.float32}:
        dw_all, dw = within(V, D, dw_kind, 7.0)
        loss = torch.empty(T, device=DEV)
        losses.head_cross_entropy(h, w, y, loss, dh, dw, workspace(losses, h, w), piece=256)
        Head(h0, w0, y).check(loss, dh, dw)
        for whole in (dh_all, dw_all):
            assert (whole[:, :shift] == 7).all() and (whole[:, shift + D:] == 7).all()


@pytest.mark.parametrize("kind", TYPES, ids=str)
def test_some_gradients_alone(losses, kind):
    h, w, y, _ = inputs(100, 128, 700, kind, seed=4)
    ref = Head(h, w, y)
    for with_dh, with_dw in ((True, False), (False, True), (False, False)):
        for piece in (0, 256):
            loss, dh, dw = outputs(h, w)
            dh, dw = dh if with_dh else None, dw if with_dw else None
            losses.head_cross_entropy(h, w, y, loss, dh, dw, workspace(losses, h, w, piece=piece), piece=piece)
            ref.check(loss, dh, dw)


@pytest.mark.parametrize("kind", [torch.bfloat16, torch.float16], ids=str)
def test_weight_gradient_into_a_flat_buffer(losses, kind):
    """The operands of 16 bits, the gradient in a flat binary32 buffer behind a tensor of odd length."""
    T, D, V = 200, 100, 333
    h, w, y, _ = inputs(T, D, V, kind, seed=5)
    flat = torch.full((17 + V * D + 5,), 3.0, device=DEV)
    dw = flat[17:17 + V * D].view(V, D)
    loss, dh, _ = outputs(h, w)
    losses.head_cross_entropy(h, w, y, loss, dh, dw, workspace(losses, h, w))
    Head(h, w, y).check(loss, dh, dw)
    assert (flat[:17] == 3).all() and (flat[-5:] == 3).all()


@pytest.mark.parametrize("kind", TYPES, ids=str)
@pytest.mark.parametrize("spread", [1e-3, 30.0])
def test_flat_and_peaked_logits(losses, kind, spread):
    h, w, y, _ = inputs(150, 64, 900, kind, seed=6, spread=spread)
    loss, dh, dw = outputs(h, w)
    losses.head_cross_entropy(h, w, y, loss, dh, dw, workspace(losses, h, w, piece=512), piece=512)
    Head(h, w, y).check(loss, dh, dw)


@pytest.mark.parametrize("scales", [(1e-20, 1e15), (1e18, 1e-16), (1e-30, 1e-8)], ids=str)
def test_binary32_ranges(losses, scales):
    """Operands far from one: their halves are scaled, not clipped."""
    h, w, y, _ = inputs(80, 96, 500, torch.float32, seed=7)
    h, w = h * scales[0], w * scales[1]
    loss, dh, dw = outputs(h, w)
    losses.head_cross_entropy(h, w, y, loss, dh, dw, workspace(losses, h, w))
    Head(h, w, y).check(loss, dh, dw)


@pytest.mark.parametrize("kind", TYPES, ids=str)
def test_small_weights_keep_their_gradient(losses, kind):
    """Tokens whose weights differ by thousands: the gradient is stored relative to the largest."""
    h, w, y, gen = inputs(130, 64, 400, kind, seed=8)
    weight = 10.0 ** (-4 * torch.rand(130, generator=gen, device=DEV))
    loss, dh, dw = outputs(h, w)
    losses.head_cross_entropy(h, w, y, loss, dh, dw, workspace(losses, h, w), weight=weight, scale=2.0 ** -3)
    Head(h, w, y, weight=weight, scale=2.0 ** -3).check(loss, dh, dw)


def top_of(T, V, top, gen):
    index = torch.stack([torch.randperm(V, generator=gen, device=DEV)[:top] for _ in range(T)]).to(torch.int32)
    logit = 3.0 * torch.randn(T, top, generator=gen, device=DEV)
    return index, logit


@pytest.mark.parametrize("kind", TYPES, ids=str)
@pytest.mark.parametrize("size", [(1, 1, 1, 1), (1, 24, 90, 7), (33, 64, 300, 1), (100, 136, 1000, 64), (261, 72, 800, 130)], ids=str)
@pytest.mark.parametrize("mix", [(0.0, 1.0, 1.0), (0.4, 0.6, 2.0), (1.0, -0.5, 0.7)], ids=str)
def test_distill(losses, size, mix, kind):
    T, D, V, top = size
    hard, soft, t = mix
    h, w, y, gen = inputs(T, D, V, kind, seed=9)
    index, logit = top_of(T, V, top, gen)
    loss, dh, dw = outputs(h, w)
    losses.head_distill(h, w, index, logit, loss, dh, dw, workspace(losses, h, w, top=top), temperature=t, soft=soft,
                        target=y if hard else None, hard=hard, scale=1.0 / T)
    Head(h, w, y if hard else None, index, logit, t, hard, soft, scale=1.0 / T).check(loss, dh, dw)


@pytest.mark.parametrize("kind", TYPES, ids=str)
@pytest.mark.parametrize("piece", [0, 256])
def test_distill_entries(losses, kind, piece):
    """Entries left out by their index or a logit of -inf, entries that occur twice, entries that are the label, tokens without any."""
    T, D, V, top = 210, 88, 700, 20
    h, w, y, gen = inputs(T, D, V, kind, seed=10)
    index, logit = top_of(T, V, top, gen)
    index[::4, 3] = -1
    index[1::4, 0] = V
    logit[2::4, 5:9] = float("-inf")
    index[::5, 7] = index[::5, 2]                       # twice
    index[::5, 8] = index[::5, 2]                       # three times
    index[::3, 1] = y[::3]                              # the label among them
    logit[10:20] = float("-inf")                        # none left
    index[20:30] = -7
    y[15:25] = -1                                       # some of those have no label either
    y[100:110] = -1
    weight = torch.rand(T, generator=gen, device=DEV) + 0.1
    weight[50:60] = 0.0
    clean = h.clone()
    ref = Head(clean, w, y, index, logit, 2.0, 0.5, 0.5, weight, 0.5)
    assert not ref.counts[15:25].any() and ref.counts[10:15].all() and ref.counts[100:110].all()
    h[~ref.counts] = float("nan")
    logit[50:60] = float("nan")
    loss, dh, dw = outputs(h, w)
    losses.head_distill(h, w, index, logit, loss, dh, dw, workspace(losses, h, w, top=top, piece=piece), temperature=2.0, soft=0.5,
                        target=y, hard=0.5, weight=weight, scale=0.5, piece=piece)
    ref.check(loss, dh, dw)


@pytest.mark.parametrize("kind", TYPES, ids=str)
def test_distilling_from_itself(losses, kind):
    """A teacher whose entries are the whole vocabulary and the head's own logits: no loss, no gradient to speak of."""
    T, D, V = 40, 64, 96
    h, w, _, _ = inputs(T, D, V, kind, seed=11)
    index = torch.arange(V, device=DEV, dtype=torch.int32).repeat(T, 1)
    logit = (h.double() @ w.double().t()).float()
    loss, dh, dw = outputs(h, w)
    losses.head_distill(h, w, index, logit, loss, dh, dw, workspace(losses, h, w, top=V), temperature=1.5)
    Head(h, w, None, index, logit, 1.5, 0.0, 1.0).check(loss, dh, dw)


@pytest.mark.parametrize("mix", [(1.0, 0.0), (0.3, 0.7)], ids=str)
def test_gradient_against_differences(losses, mix):
    """<gradient, direction> against the loss's own central difference.  The loss of a token is smooth on the scale of a logit:
    its third derivative along a direction that moves every logit by about one is below 2, so a step of 2^-6 leaves less than 2^-12 of
    it; losses are off by less than 2^-18 each, which the step turns into 2^-12."""
    hard, soft = mix
    T, D, V, top = 24, 64, 200, 16
    h, w, y, gen = inputs(T, D, V, torch.float32, seed=12)
    index, logit = top_of(T, V, top, gen)
    vh, vw = torch.randn(T, D, generator=gen, device=DEV) / D ** 0.5 / 3, torch.randn(V, D, generator=gen, device=DEV) / D ** 0.5 / 3

    def call(h, w):
        loss, dh, dw = outputs(h, w)
        losses.head_distill(h, w, index, logit, loss, dh, dw, workspace(losses, h, w, top=top), temperature=2.0, soft=soft, target=y, hard=hard)
        return loss.double().sum().item(), dh, dw

    _, dh, dw = call(h, w)
    step = 2.0 ** -6
    for v, u in ((vh, 0 * vw), (0 * vh, vw), (vh, vw)):
        up, down = call(h + step * v, w + step * u)[0], call(h - step * v, w - step * u)[0]
        slope = (dh.double() * v).sum().item() + (dw.double() * u).sum().item()
        assert abs((up - down) / (2 * step) - slope) <= T * 4 * (2.0 ** -12 + 2.0 ** -12), (up, down, slope)


@pytest.mark.parametrize("kind", TYPES, ids=str)
def test_same_bytes_on_another_stream_and_in_a_graph(losses, kind):
    T, D, V, top = 150, 128, 1200, 12
    h, w, y, gen = inputs(T, D, V, kind, seed=13)
    index, logit = top_of(T, V, top, gen)
    ws = workspace(losses, h, w, top=top, piece=512)

    def call(out, stream=None):
        losses.head_distill(h, w, index, logit, *out, ws, temperature=2.0, soft=0.5, target=y, hard=0.5, piece=512, stream=stream)

    first = outputs(h, w)
    call(first)
    second = outputs(h, w)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    call(second, side)
    torch.cuda.synchronize()
    third = outputs(h, w)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        call(third)
    for _ in range(3):
        for x in third:
            x.fill_(float("nan"))
        ws.fill_(0xFF)
        graph.replay()
        torch.cuda.synchronize()
        for a, b, c in zip(first, second, third):
            assert torch.equal(a, b) and torch.equal(a, c)


def test_a_head_larger_than_32_bits(losses):
    """Weight and gradient of more than 2^31 elements: labels at both ends, few tokens."""
    T, D, V = 3, 1032, 2_100_000
    w = torch.zeros(V, D, dtype=torch.bfloat16, device=DEV)
    h = torch.randn(T, D, generator=torch.Generator(device=DEV).manual_seed(3), device=DEV).to(torch.bfloat16)
    last = V - 1
    w[last] = h[0]
    w[0] = h[1]
    y = torch.tensor([last, 0, 5], dtype=torch.int32, device=DEV)
    loss, dh = torch.empty(T, device=DEV), torch.empty_like(h)
    dw = torch.empty_like(w)
    losses.head_cross_entropy(h, w, y, loss, dh, dw, workspace(losses, h, w, piece=300_000), piece=300_000)
    z = h.double() @ torch.stack([w[0], w[last]]).double().t()          # all other logits are 0
    rest = torch.full((T, 1), float(V - 2), dtype=torch.float64, device=DEV).log()
    lse = torch.logsumexp(torch.cat([z, rest], 1), 1)
    want = lse - torch.stack([z[0, 1], z[1, 0], torch.zeros_like(z[0, 0])])
    assert torch.allclose(loss.double(), want, rtol=1e-5, atol=2e-3)
    p = (z - lse[:, None]).exp()
    for row, column, t in ((0, 0, 1), (last, 1, 0)):
        g = p[:, column].clone()
        g[t] -= 1
        assert torch.allclose(dw[row].double(), g @ h.double(), rtol=2.0 ** -6, atol=2.0 ** -6)
    g = (-lse).exp()
    g[2] -= 1
    assert torch.allclose(dw[5].double(), g @ h.double(), rtol=2.0 ** -6, atol=2.0 ** -6)
    middle = dw[V // 2 + 77].double()                                   # p of exp(-lse) each
    assert torch.allclose(middle, (-lse).exp() @ h.double(), rtol=2.0 ** -6, atol=1e-9)
