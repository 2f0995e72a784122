"""The router on the GPU against its formulas in 64 bits.

Choices and counts are whole numbers and equal. Tolerances of the others: a score less the row's highest is rounded once, off by 2^-24 of itself, which
the exponential turns into a share of its value; expf itself is granted 4 roundings; a row's sum of E terms is within E 2^-24. `off(E, far)`, with `far` the largest such
difference, is the share that a probability may be off by: E + 16 + 2 far roundings. The balance loss sums as many such probabilities as there are rows and experts;
a score's gradient is p (g - sum p g), each part of which is granted what its probabilities are off by and a rounding for each of its terms."""
import pytest

from tests.gpu_common import say
from tests.test_gpu_features import BF16, F16, F32, TYPES, U, close, generator, normal, strided

pytestmark = pytest.mark.gpu
torch = pytest.importorskip("torch")
INF = float("inf")


@pytest.fixture(scope="module")
def ctx():
    from paper_2506_22668_amd import Context
    c = Context("cuda:0")
    yield c
    c.close()


def exact_route(x, k, renorm):
    x = x.double()
    rows, experts = x.shape
    some = x.amax(1) > -INF
    top = torch.where(some, x.amax(1), 0.0)[:, None]
    q = torch.exp(x - top)
    p = torch.where(some[:, None], q / q.sum(1, keepdim=True).clamp(min=1e-300), 0.0)
    held, order = torch.sort(x, dim=1, descending=True, stable=True)
    ids = torch.where(held[:, :k] > -INF, order[:, :k], -1)
    w = torch.where(ids >= 0, p.gather(1, ids.clamp(min=0)), 0.0)
    if renorm:
        w = torch.where(some[:, None], w / w.sum(1, keepdim=True).clamp(min=1e-300), 0.0)
    counts = torch.stack([(ids == e).sum() for e in range(experts)] + [some.sum()])
    loss = experts * (counts[:experts].double() * p.sum(0)).sum() / counts[:experts].sum().clamp(min=1) / counts[experts].clamp(min=1)
    lse = torch.where(some, top[:, 0] + torch.log(q.sum(1)), -INF)
    return ids.t(), w.t(), counts, loss, lse, p


def far_of(x):
    """The largest difference of a row's finite scores (per row)."""
    x = x.double()
    return torch.where(torch.isfinite(x), x.amax(1, keepdim=True) - x, 0.0).amax(1).clamp(min=0)


def off(x):
    return (x.shape[1] + 16 + 2 * far_of(x)) * U


def gradient_exact(x, lse, ids, counts, dw, dloss, renorm):
    """(gradient, a bound of its parts' magnitudes, what it may be off by however small it is) in 64 bits."""
    x, ids = x.double(), ids.long()
    experts = x.shape[1]
    some = lse > -INF
    p = torch.where(some[:, None], torch.exp(x - torch.where(some, lse.double(), 0.0)[:, None]), 0.0)
    g = torch.zeros_like(x)
    if dloss is not None:
        g += dloss.double() * experts * counts[:experts].double() / counts[:experts].sum().clamp(min=1) / counts[experts].clamp(min=1)
    size = g.abs()
    if dw is not None:
        held = (ids >= 0).double()
        dp, big = dw.double() * held, dw.double().abs() * held
        if renorm:
            w = p.gather(1, ids.clamp(min=0).t()).t() * held
            total = torch.where(some, w.sum(0), 1.0)
            dp, big = held * (dp - (dp * w).sum(0) / total) / total, held * (big + (big * w).sum(0) / total) / total
        at = ids.clamp(min=0).t()
        g, size = g.scatter_add(1, at, dp.t()), size.scatter_add(1, at, big.t())
    by = size + (p * size).sum(1, keepdim=True)
    # (below 2^-126 the 4 roundings of the exponential are of up to 2^-150 each, whatever its value)
    return p * (g - (p * g).sum(1, keepdim=True)), p * by, 4 * 2.0 ** -150 * by


def scores(g, rows, experts, t, closed=0.0, padded=0.0, spread=1.0):
    x = normal(g, rows, experts, t=t, scale=spread)
    x[torch.rand(rows, experts, generator=g, device="cuda") < closed] = -INF
    x[torch.rand(rows, generator=g, device="cuda") < padded] = -INF
    return x


def check(ctx, g, x, k, renorm):
    rows, experts = x.shape
    ids, w, counts, loss, lse = ctx.route(x, k, renorm=renorm)
    ei, ew, ec, el, else_, p = exact_route(x, k, renorm)
    assert ids.dtype == torch.int32 and torch.equal(ids.long(), ei)
    assert counts.dtype == torch.int64 and torch.equal(counts, ec)
    share = off(x) + (3 + k) * U
    # (below 2^-126 a rounding is off by up to 2^-150, whatever the value: exponential, its share of the sum, and that of the chosen, which multiplies by E at the most)
    close(w, ew, 2 * share * ew + 3 * experts * 2.0 ** -150)
    some = else_ > -INF
    assert torch.equal(lse > -INF, some)
    if some.any():
        close(lse[some], else_[some], share[some] + 2 * U * else_[some].abs() + U * x[some].double().amax(1).abs())
    close(loss, el, (off(x).max() + (rows + experts + 8) * U) * el)
    again = ctx.route(x, k, renorm=renorm)
    assert all(torch.equal(a, b) for a, b in zip((ids, w, counts, loss, lse), again))
    dw, dloss = normal(g, k, rows), normal(g, 1) * 50
    for a, b in [(dw, dloss[0]), (dw, None), (None, dloss)]:
        dx = ctx.route_backward(x, lse, ids, counts, dweights=a, dloss=b, renorm=renorm)
        e, size, least = gradient_exact(x, lse, ids, counts, a, b, renorm)
        share = (2 * experts + 64 + 8 * (far_of(x) + lse.double().abs().where(some, 0.0)) + 4 * k)[:, None] * U
        assert dx.dtype == x.dtype
        close(dx, e, share * size + least)
        assert not dx[~some].any()
        assert torch.equal(dx, ctx.route_backward(x, lse, ids, counts, dweights=a, dloss=b, renorm=renorm))


EXPERTS = [1, 2, 3, 4, 7, 8, 9, 15, 16, 17, 31, 33, 64, 65, 100, 128, 129, 256, 257, 513, 1000, 1023, 1024]


@pytest.mark.parametrize("t", TYPES)
@pytest.mark.parametrize("experts", EXPERTS)
def test_route(ctx, t, experts):
    say(f"route {t} experts={experts}")
    g = generator(experts)
    for rows, pad, shift, closed, padded, k, renorm in [(1, 0, 0, 0.0, 0.0, 1, False), (37, 3, 1, 0.3, 0.2, 8, True), (301, 0, 0, 0.0, 0.1, 2, True),
                                                        (130, 1, 0, 0.9, 0.0, 3, False), (65, 0, 0, 1.0, 0.0, 2, True)]:
        check(ctx, g, strided(scores(g, rows, experts, t, closed, padded), pad, shift), min(k, experts), renorm)


@pytest.mark.parametrize("t", TYPES)
@pytest.mark.parametrize("k", [1, 2, 3, 4, 5, 6, 7, 8])
def test_route_numbers_of_experts_to_a_row(ctx, t, k):
    say(f"route {t} k={k}")
    g = generator(k)
    for experts in (8, 40):
        check(ctx, g, scores(g, 100, experts, t, 0.2, 0.1), k, k % 2 == 0)


@pytest.mark.parametrize("t", TYPES)
@pytest.mark.parametrize("rows, experts, k", [(70_001, 8, 2), (40_003, 64, 1), (20_011, 300, 4)])
def test_route_many_rows(ctx, t, rows, experts, k):
    say(f"route many rows {t} rows={rows} experts={experts}")
    g = generator(rows)
    check(ctx, g, scores(g, rows, experts, t, 0.0, 0.01), k, True)


@pytest.mark.parametrize("t", TYPES)
def test_route_far_scores(ctx, t):
    """Scores hundreds apart, and the lowest values of their type: those are open, -inf alone is closed."""
    say(f"route far scores {t}")
    g = generator(11)
    check(ctx, g, scores(g, 200, 24, t, 0.1, 0.1, spread=60.0), 4, True)
    low = torch.finfo(t).min
    x = torch.full((3, 5), low, dtype=t, device="cuda")
    x[1, 3], x[2, :] = 0.0, -INF
    ids, w, counts, loss, lse = ctx.route(x, 2)
    assert ids.tolist() == [[0, 3, -1], [1, 0, -1]] and counts.tolist() == [2, 1, 0, 1, 0, 2]
    # (equal scores, far = 0: the share of the module's bound, in the weight and in the sum; 1/5 itself is no fp32 number)
    close(w[:, 0], torch.full((2,), 0.2, dtype=torch.float64, device="cuda"), 2 * (5 + 16 + 3 + 2) * U * 0.2)
    assert w[0, 1] == 1 and w[1, 1] == 0 and not w[:, 2].any()


@pytest.mark.parametrize("t", TYPES)
def test_route_ties_go_to_the_lowest_expert(ctx, t):
    say(f"route ties {t}")
    for experts in (6, 64, 700):
        x = torch.zeros(5, experts, dtype=t, device="cuda")
        x[1, 1::2] = -0.0                       # (equal to 0)
        x[2, experts - 1] = x[2, 2] = 1.0
        x[3, :3] = -INF
        k = 4
        ids = ctx.route(x, k)[0].t().tolist()
        assert ids == [[0, 1, 2, 3], [0, 1, 2, 3], [2, experts - 1, 0, 1], [3, 4, 5, 6] if experts > 6 else [3, 4, 5, -1], [0, 1, 2, 3]]


@pytest.mark.parametrize("t", TYPES)
@pytest.mark.parametrize("bad", [INF, float("nan")])
def test_rows_that_are_not_finite_have_no_expert(ctx, t, bad):
    say(f"route {bad} {t}")
    g = generator(12)
    for experts in (5, 70, 300):
        x = scores(g, 40, experts, t)
        want = ctx.route(x, 2, renorm=True)
        x[7, experts - 1], x[9, 0] = bad, bad
        x[9, 1:] = -INF
        ids, w, counts, loss, lse = ctx.route(x, 2, renorm=True)
        rest = [i for i in range(40) if i not in (7, 9)]
        assert torch.equal(ids[:, rest], want[0][:, rest]) and torch.equal(w[:, rest], want[1][:, rest]) and torch.equal(lse[rest], want[4][rest])
        for r in (7, 9):
            assert (ids[:, r] == -1).all() and torch.isnan(w[:, r]).all() and torch.isnan(lse[r])
        assert torch.isnan(loss) and counts[experts] == 38 and counts[:experts].sum() == 76
        dx = ctx.route_backward(x, lse, ids, counts, dweights=torch.ones(2, 40, device="cuda"), renorm=True)
        assert torch.isnan(dx[7]).all() and torch.isnan(dx[9]).all() and torch.isfinite(dx[rest]).all()


@pytest.mark.parametrize("t", TYPES)
def test_route_without_rows_and_one_row_for_all(ctx, t):
    say(f"route without rows {t}")
    x = torch.empty(0, 6, dtype=t, device="cuda")
    ids, w, counts, loss, lse = ctx.route(x, 2)
    assert ids.shape == (2, 0) and w.shape == (2, 0) and lse.shape == (0,) and not counts.any() and loss == 0
    assert ctx.route_backward(x, lse, ids, counts, dweights=w).shape == (0, 6)
    one = normal(generator(13), 1, 6, t=t)
    a, b = ctx.route(one.expand(90, 6), 2), ctx.route(one.repeat(90, 1), 2)
    assert all(torch.equal(p, q) for p, q in zip(a, b))
    assert torch.equal(ctx.route(one.repeat(90, 1).t().contiguous().t(), 2)[1], b[1])


def test_even_use_has_a_loss_of_one(ctx):
    say("route even use")
    x = torch.zeros(64, 8, device="cuda")
    x[torch.arange(64), torch.arange(64) % 8] = 3.0
    _, _, counts, loss, _ = ctx.route(x, 1)
    assert (counts[:8] == 8).all() and abs(loss.item() - 1) < 64 * U
    all_one = torch.zeros(64, 8, device="cuda")
    all_one[:, 2] = 80.0
    assert abs(ctx.route(all_one, 1)[3].item() - 8) < 8 * 200 * U


@pytest.mark.parametrize("renorm", [False, True])
def test_route_gradient_against_differences(ctx, renorm):
    """sum(c w) + d loss of the choices as they stand, moved by +-h along a direction, in 64 bits: the third-order rest of the difference is below h^2 times
    the size of the parts (each derivative of a softmax by a direction of size 1 at most triples)."""
    say(f"route differences renorm={renorm}")
    g = generator(14)
    x = scores(g, 60, 9, F32, 0.1, 0.1)
    ids, _, counts, _, lse = ctx.route(x, 3, renorm=renorm)
    c, d, v = normal(g, 3, 60), normal(g, 1), torch.rand(60, 9, generator=g, device="cuda") * 2 - 1
    grad = ctx.route_backward(x, lse, ids, counts, dweights=c, dloss=d, renorm=renorm)

    def value(z):
        some = z.amax(1) > -INF
        p = torch.where(some[:, None], torch.softmax(torch.where(some[:, None], z, 0.0), 1), 0.0)
        w = torch.where(ids >= 0, p.gather(1, ids.long().clamp(min=0).t()).t(), 0.0)
        if renorm:
            w = torch.where(some, w / torch.where(some, w.sum(0), 1.0), 0.0)
        loss = 9 * (counts[:9].double() * p.sum(0)).sum() / counts[:9].sum() / counts[9]
        return (w * c.double()).sum() + loss * d.double()[0]
    h = 1e-4
    slope = (value(x.double() + h * v.double()) - value(x.double() - h * v.double())) / (2 * h)
    parts = (c.double().abs().sum() + 9 * d.double().abs()[0])
    assert abs(slope - (grad.double() * v.double()).sum()) <= 27 * h * h * parts + 400 * U * parts


@pytest.mark.parametrize("t, element", [(F32, 0), (BF16, 1), (F16, 2)])
def test_route_outputs_with_rows_apart_and_in_place(ctx, t, element):
    say(f"route strided {t}")
    import ctypes as C
    lib, g = ctx.lib, generator(15)
    rows, experts, pad, k = 67, 53, 5, 2
    x = scores(g, rows, experts, t, 0.1, 0.1)
    ids, w, counts, loss, lse = ctx.route(x, k)
    dw = normal(g, k, rows)
    want = ctx.route_backward(x, lse, ids, counts, dweights=dw)
    out = torch.full((rows, experts + pad), 3.0, dtype=t, device="cuda")
    args = lambda to, step, frm: (ctx.h, element, rows, experts, k, 0, frm.data_ptr(), step if frm is to else experts, lse.data_ptr(), ids.data_ptr(),   # noqa: E731
                                  counts.data_ptr(), dw.data_ptr(), None, to.data_ptr(), step)
    assert lib.ds_route_backward(*args(out, experts + pad, x)) == 0
    assert torch.equal(out[:, :experts], want) and (out[:, experts:] == 3).all()
    here = x.clone()
    assert lib.ds_route_backward(*args(here, experts, here)) == 0
    assert torch.equal(here, want)
    need = C.c_int64()
    assert lib.ds_route_workspace(rows, experts, C.byref(need)) == 0
    ws = torch.full((need.value + 64,), 77, dtype=torch.uint8, device="cuda")
    i2, w2, c2, l2 = torch.empty_like(ids), torch.empty_like(w), torch.empty_like(counts), torch.empty_like(loss)
    assert lib.ds_route(ctx.h, element, rows, experts, k, 0, x.data_ptr(), experts, i2.data_ptr(), w2.data_ptr(), c2.data_ptr(), l2.data_ptr(), None, ws.data_ptr(),
                        need.value) == 0     # (an inference keeps no lse)
    assert torch.equal(i2, ids) and torch.equal(w2, w) and torch.equal(c2, counts) and torch.equal(l2, loss) and (ws[need.value:] == 77).all()
    # ids and counts that are out of range lead nowhere
    wild = ids.clone()
    wild[0, 0], wild[1, 1], wild[0, 2] = experts, -7, 2 ** 31 - 1
    got = ctx.route_backward(x, lse, wild, counts, dweights=dw, renorm=True)
    rest = [i for i in range(rows) if i > 2]
    assert torch.equal(got[rest], ctx.route_backward(x, lse, ids, counts, dweights=dw, renorm=True)[rest])
    torch.cuda.synchronize()
