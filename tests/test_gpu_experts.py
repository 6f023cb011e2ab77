"""The experts' products and their gradients against their definitions in 64 bits."""
import pytest
import torch

from layer_reference import Experts

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
TYPES = [torch.float32, torch.bfloat16, torch.float16]
# tokens, slots, experts, in, out
SIZES = [(1, 1, 1, 1, 1), (1, 2, 8, 64, 128), (1, 8, 64, 256, 192), (7, 3, 5, 33, 17), (63, 2, 4, 100, 70), (64, 1, 1, 128, 256), (65, 1, 1, 129, 257),
         (200, 2, 8, 48, 96), (333, 2, 8, 513, 640), (300, 4, 100, 72, 40), (1000, 3, 4, 320, 200), (129, 6, 1024, 16, 24), (2048, 2, 4, 512, 1024),
         (2600, 2, 4, 192, 4096), (2300, 2, 4, 4096, 200)]


@pytest.fixture(scope="module")
def experts(gpu_lib):
    from paper_1901_01544_amd import experts
    return experts


def inputs(T, K, E, D, F, kind, by_slot=False, nobody=0.1, seed=0):
    gen = torch.Generator(device=DEV).manual_seed(seed * 7919 + T * 31 + D)
    x = torch.randn((T, K, D) if by_slot else (T, D), generator=gen, device=DEV).to(kind)
    w = (D ** -0.5 * torch.randn(E, F, D, generator=gen, device=DEV)).to(kind)
    dy = torch.randn(T, K, F, generator=gen, device=DEV).to(kind)
    chosen = torch.rand(T, E, generator=gen, device=DEV).topk(K, dim=1).indices.to(torch.int32)
    chosen = torch.where(torch.rand(T, K, generator=gen, device=DEV) < nobody, -1, chosen)
    return x, w, chosen, dy


def workspace(experts, x, w, chosen, gradient):
    return torch.full((experts.product_workspace_bytes(x, w, chosen, gradient=gradient),), 0xFF, dtype=torch.uint8, device=DEV)


def product(experts, x, w, chosen, y=None):
    if y is None:
        y = torch.full((*chosen.shape, w.shape[1]), float("nan"), dtype=x.dtype, device=DEV)
    experts.product(x, w, chosen, y, workspace(experts, x, w, chosen, False))
    return y


def gradient(experts, x, w, chosen, dy, dw_kind=None, dx=True, dw=True):
    dx = torch.full(x.shape, float("nan"), dtype=x.dtype, device=DEV) if dx is True else dx
    dw = torch.full(w.shape, float("nan"), dtype=dw_kind or w.dtype, device=DEV) if dw is True else dw
    experts.product_gradient(x, w, chosen, dy, dx, dw, workspace(experts, x, w, chosen, True))
    return dx, dw


@pytest.mark.parametrize("kind", TYPES, ids=str)
@pytest.mark.parametrize("size", SIZES, ids=str)
@pytest.mark.parametrize("by_slot", [False, True])
def test_product_and_gradient(experts, size, kind, by_slot):
    x, w, chosen, dy = inputs(*size, kind, by_slot)
    ref = Experts(x, w, chosen, dy)
    ref.check(product(experts, x, w, chosen))
    ref.check_gradient(*gradient(experts, x, w, chosen, dy))
    ref.check_gradient(*gradient(experts, x, w, chosen, dy, dw_kind=torch.float32))


@pytest.mark.parametrize("kind", TYPES, ids=str)
def test_uneven_experts(experts, kind):
    """One expert has most of the rows, some have none, one has as many as fill its tiles, one a row more."""
    x, w, _, dy = inputs(1500, 2, 9, 192, 160, kind)
    flat = torch.zeros(3000, dtype=torch.int32, device=DEV)
    flat[:256], flat[256:513], flat[513:514], flat[514:578] = 3, 8, 5, 2
    gen = torch.Generator(device=DEV).manual_seed(1)
    chosen = flat[torch.randperm(3000, generator=gen, device=DEV)].view(1500, 2)
    ref = Experts(x, w, chosen, dy)
    ref.check(product(experts, x, w, chosen))
    dx, dw = gradient(experts, x, w, chosen, dy)
    ref.check_gradient(dx, dw)
    assert all((dw[e] == 0).all() for e in (1, 4, 6, 7))


@pytest.mark.parametrize("kind", TYPES, ids=str)
@pytest.mark.parametrize("by_slot", [False, True])
@pytest.mark.parametrize("size,nobody", [((700, 4, 8, 96, 130), 0.875), ((3000, 4, 8, 129, 96), 0.875), ((9000, 2, 4, 128, 2304), 0.7), ((2500, 1, 2, 64, 333), 0.9)], ids=str)
def test_most_slots_are_nobodys(experts, size, nobody, kind, by_slot):
    """As where a rank has an eighth of the experts, with small, middling and large tiles: zeros behind the experts' tiles, in every row of nobody."""
    x, w, chosen, dy = inputs(*size, kind, by_slot, nobody)
    ref = Experts(x, w, chosen, dy)
    y = product(experts, x, w, chosen)
    ref.check(y)
    assert (y[chosen < 0] == 0).all()
    dx, dw = gradient(experts, x, w, chosen, dy)
    ref.check_gradient(dx, dw)
    assert (dx[(chosen < 0) if by_slot else (chosen < 0).all(1)] == 0).all()


@pytest.mark.parametrize("kind", TYPES, ids=str)
@pytest.mark.parametrize("by_slot", [False, True])
def test_no_rows_at_all(experts, kind, by_slot):
    x, w, chosen, dy = inputs(40, 2, 6, 64, 80, kind, by_slot)
    x.fill_(float("nan")), w.fill_(float("nan")), dy.fill_(float("nan"))
    chosen[::2], chosen[1::2] = -1, 6
    assert (product(experts, x, w, chosen) == 0).all()
    dx, dw = gradient(experts, x, w, chosen, dy)
    assert (dx == 0).all() and (dw == 0).all()
    empty = x[:0], w, chosen[:0]
    assert product(experts, *empty).shape == (0, 2, 80)
    dx, dw = gradient(experts, *empty, dy[:0])
    assert dx.shape == x[:0].shape and (dw == 0).all()


@pytest.mark.parametrize("kind", TYPES, ids=str)
@pytest.mark.parametrize("by_slot", [False, True])
@pytest.mark.parametrize("T,D", [(150, 72), (150, 128), (20, 72)])
def test_nan_and_infinity_stay_with_their_rows(experts, kind, by_slot, T, D):
    K, E, F = 2, 5, 136
    x, w, chosen, dy = inputs(T, K, E, D, F, kind, by_slot, nobody=0.2)
    chosen[chosen == 4] = 3                                             # nobody's matrix
    clean = Experts(x, w, chosen, dy)
    bad, inf = float("nan"), float("inf")
    w[4] = bad
    w[2, 7, 5] = bad
    w[1, F - 1, D - 1] = inf
    x.view(-1, D)[-1, 3] = -inf
    dy[chosen < 0] = bad
    dy[17, 0, 9] = inf
    y = product(experts, x, w, chosen)
    dx, dw = gradient(experts, x, w, chosen, dy)
    ref = Experts(x, w, chosen, torch.where((chosen < 0)[:, :, None], 0.0, dy.float()).to(kind))
    for got, want, was, off in ((y, ref.y, clean.y, clean.y_off), (dx, ref.dx, clean.dx, clean.dx_off), (dw, ref.dw, clean.dw, clean.dw_off)):
        assert not torch.isfinite(got[~torch.isfinite(want)]).any() and got[want.isnan()].isnan().all()
        there = torch.isfinite(want)
        assert torch.isfinite(got[there]).all() and torch.equal(want[there], was[there])


@pytest.mark.parametrize("kind", TYPES, ids=str)
@pytest.mark.parametrize("shift,more", [(0, 8), (1, 3), (8, 16), (4, 5)])
@pytest.mark.parametrize("T", [10, 90])
def test_strides_and_alignments(experts, kind, shift, more, T):
    """Rows of every matrix a stretch of longer ones, matrices apart from each other; what lies around the outputs stays."""
    K, E, D, F = 3, 4, 96, 56
    for by_slot in (False, True):
        x0, w0, chosen, dy0 = inputs(T, K, E, D, F, kind, by_slot)

        def within(t, fill):
            rows = t.reshape(-1, t.shape[-1])
            whole = torch.full((rows.shape[0] + 2, rows.shape[1] + shift + more), fill, dtype=t.dtype, device=DEV)
            part = whole[1:-1, shift:shift + rows.shape[1]]
            part.copy_(rows)
            return whole, part.unflatten(0, t.shape[:-1])

        nan = float("nan")
        x, dy = within(x0, nan)[1], within(dy0, nan)[1]
        apart = torch.full((E, F + 3, D + shift + more), nan, dtype=kind, device=DEV)
        w = apart[:, 2:2 + F, shift:shift + D]
        w.copy_(w0)
        ref = Experts(x0, w0, chosen, dy0)
        whole_y, y = within(torch.zeros_like(dy0), 9.0)
        whole_dx, dx = within(torch.zeros_like(x0), 9.0)
        for dw_kind in {kind, torch.float32}:
            apart_dw = torch.full((E, F + 3, D + shift + more), 9.0, dtype=dw_kind, device=DEV)
            dw = apart_dw[:, 2:2 + F, shift:shift + D]
            product(experts, x, w, chosen, y)
            gradient(experts, x, w, chosen, dy, dx=dx, dw=dw)
            ref.check(y)
            ref.check_gradient(dx, dw)
            for whole, part in ((whole_y, y), (whole_dx, dx), (apart_dw, dw)):
                n = part.numel()
                assert (whole == 9.0).sum() >= whole.numel() - n
                part.fill_(9.0)
                assert (whole == 9.0).all()


def test_one_of_the_gradients(experts):
    for by_slot in (False, True):
        x, w, chosen, dy = inputs(200, 2, 6, 128, 64, torch.bfloat16, by_slot)
        dx, dw = gradient(experts, x, w, chosen, dy)
        assert torch.equal(gradient(experts, x, w, chosen, dy, dw=None)[0], dx)
        assert torch.equal(gradient(experts, x, w, chosen, dy, dx=None)[1], dw)


def test_an_expert_for_two_slots_of_a_token(experts):
    x, w, chosen, dy = inputs(80, 3, 4, 40, 48, torch.float32)
    chosen[:, 1] = chosen[:, 0]
    ref = Experts(x, w, chosen, dy)
    ref.check(product(experts, x, w, chosen))
    ref.check_gradient(*gradient(experts, x, w, chosen, dy))


def test_matrices_gradient_in_a_flat_buffer(experts):
    """As the compression step takes it: a view that begins at an odd element."""
    x, w, chosen, dy = inputs(150, 2, 5, 77, 31, torch.bfloat16)
    flat = torch.full((3 + w.numel() + 9,), 9.0, device=DEV)
    dw = flat[3:3 + w.numel()].view(w.shape)
    Experts(x, w, chosen, dy).check_gradient(*gradient(experts, x, w, chosen, dy, dw=dw))
    assert (flat[:3] == 9).all() and (flat[3 + w.numel():] == 9).all()


def test_gradient_against_differences(experts):
    """The product is linear in x and in w, so a difference over any step is the slope but for the sums' rounding: y of about 1, with
    sums of 48 or 30 terms off by 2^-20 of their size, a step of 1."""
    x, w, chosen, dy = inputs(60, 2, 5, 48, 30, torch.float32)
    gen = torch.Generator(device=DEV).manual_seed(3)
    vx, vw = torch.randn(x.shape, generator=gen, device=DEV), torch.randn(w.shape, generator=gen, device=DEV)
    dx, dw = gradient(experts, x, w, chosen, dy)

    def value(x, w):
        return (product(experts, x, w, chosen).double() * dy).sum().item()

    def reach(x, w):
        return Experts(x.abs(), w.abs(), chosen).y.mul(dy.abs()).sum().item()

    for slope, at, size in ((dx.double() * vx).sum().item(), (lambda s: value(x + s * vx, w)), reach(x.abs() + vx.abs(), w)), \
                           ((dw.double() * vw).sum().item(), (lambda s: value(x, w + s * vw)), reach(x, w.abs() + vw.abs())):
        assert abs((at(1.0) - at(-1.0)) / 2 - slope) <= 3 * 2.0 ** -20 * size


@pytest.mark.parametrize("size", [(1, 4, 16, 256, 128), (70, 2, 8, 100, 60), (3000, 2, 8, 512, 512)], ids=str)
def test_same_bytes_on_another_stream_and_in_a_graph(experts, size):
    x, w, chosen, dy = inputs(*size, torch.bfloat16)

    def both(y, dx, dw, ws):
        experts.product(x, w, chosen, y, ws)
        experts.product_gradient(x, w, chosen, dy, dx, dw, ws)
        return y, dx, dw

    def empty():
        return (torch.empty_like(dy), torch.empty_like(x), torch.empty(w.shape, device=DEV),
                torch.empty(max(experts.product_workspace_bytes(x, w, chosen, gradient=g) for g in (False, True)), dtype=torch.uint8, device=DEV))

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


@pytest.mark.parametrize("T,K,E", [(2048, 1, 3), (2049, 1, 1024), (4096, 1, 3), (20000, 3, 17), (9000, 8, 64), (300_000, 1, 5)])
def test_many_slots(experts, T, K, E):
    """Several workgroups arrange them; rows so narrow that the products are nothing.  Whole numbers, so every sum is exact."""
    gen = torch.Generator(device=DEV).manual_seed(T)
    x = torch.randint(-8, 9, (T, K, 8), generator=gen, device=DEV).to(torch.bfloat16)
    w = torch.randint(-4, 5, (E, 8, 8), generator=gen, device=DEV).to(torch.bfloat16)
    chosen = torch.randint(-1, E + 1, (T, K), generator=gen, device=DEV, dtype=torch.int32)
    inside = (chosen >= 0) & (chosen < E)
    of = w.float()[torch.where(inside, chosen, 0).long()]
    want = torch.where(inside[:, :, None], (of * x.float()[:, :, None, :]).sum(3), 0.0)
    assert torch.equal(product(experts, x, w, chosen), want.to(torch.bfloat16))
    dy = torch.randint(-2, 3, (T, K, 8), generator=gen, device=DEV).to(torch.bfloat16)
    dx, dw = gradient(experts, x, w, chosen, dy, dw_kind=torch.float32)
    assert torch.equal(dx, torch.where(inside[:, :, None], (of * dy.float()[:, :, :, None]).sum(2), 0.0).to(torch.bfloat16))
    outer = dy.double()[inside][:, :, None] * x.double()[inside][:, None, :]
    want = torch.zeros(E, 8, 8, dtype=torch.float64, device=DEV).index_add_(0, chosen[inside].long(), outer)
    assert torch.equal(dw.double(), want)


@pytest.mark.parametrize("T,K,E", [(700, 2, 3), (9, 2, 3)])
def test_rows_and_matrices_far_apart(experts, T, K, E):
    """Offsets that 32 bits do not hold: rows 8 MB apart, matrices 2^31 elements."""
    D, F = 128, 64
    x0, w0, chosen, dy0 = inputs(T, K, E, D, F, torch.bfloat16, False)
    ref = Experts(x0, w0, chosen, dy0)
    far = 1 << 22

    def rows(t):
        n = t.numel() // t.shape[-1]
        part = torch.zeros(n * far, dtype=t.dtype, device=DEV).view(n, far)[:, 64:64 + t.shape[-1]]
        part.copy_(t.reshape(n, -1))
        return part.unflatten(0, t.shape[:-1]) if t.dim() == 3 else part

    def matrices(kind):
        return torch.empty((E - 1) * (1 << 31) + F * D, dtype=kind, device=DEV).as_strided((E, F, D), (1 << 31, D, 1))

    x, w = rows(x0), matrices(torch.bfloat16)
    w.copy_(w0)
    y = rows(torch.zeros_like(dy0))
    product(experts, x, w, chosen, y)
    ref.check(y.contiguous())
    y.copy_(dy0)
    dx, dw = rows(torch.zeros_like(x0)), matrices(torch.float32)
    gradient(experts, x, w, chosen, y, dx=dx, dw=dw)
    ref.check_gradient(dx.contiguous(), dw.contiguous())


def test_rows_beyond_four_gigabytes(experts):
    """More bytes of rows than 32 bits count: these are gathered.  Whole numbers, so every sum is exact."""
    T, E, D, F = 540_000, 3, 4096, 8
    gen = torch.Generator(device=DEV).manual_seed(7)
    x = torch.randint(-8, 9, (T, D), generator=gen, device=DEV, dtype=torch.int8).to(torch.bfloat16)
    w = torch.randint(-4, 5, (E, F, D), generator=gen, device=DEV).to(torch.bfloat16)
    chosen = torch.randint(-1, E, (T, 1), generator=gen, device=DEV, dtype=torch.int32)
    dy = torch.randint(-1, 2, (T, 1, F), generator=gen, device=DEV).to(torch.bfloat16)
    y = product(experts, x, w, chosen)
    dx, dw = gradient(experts, x, w, chosen, dy, dw_kind=torch.float32)
    want_dw = torch.zeros(E, F, D, dtype=torch.float64, device=DEV)
    for rows in torch.arange(T, device=DEV).split(60_000):
        part, of = x[rows].float(), chosen[rows, 0]
        for e in range(-1, E):
            mine = of == e
            if e < 0:
                assert not y[rows, 0][mine].any() and not dx[rows][mine].any()
                continue
            assert torch.equal(y[rows, 0][mine], (part[mine] @ w[e].float().t()).to(torch.bfloat16))
            assert torch.equal(dx[rows][mine], (dy[rows, 0][mine].float() @ w[e].float()).to(torch.bfloat16))
            want_dw[e] += (dy[rows, 0][mine].float().t() @ part[mine]).double()
    assert torch.equal(dw.double(), want_dw)
