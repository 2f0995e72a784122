"""The router on the GPU where scores are large, or nearly equal: the softmax of a row does not change when a number is added to all of its scores, so what is right near
0 has to be right anywhere.

Tolerances, besides those of tests/test_gpu_route.py (`off`: what a probability may be off by): a row's lse is its highest score and the logarithm of a sum that begins with 1. The sum's
share is `off`; its logarithm to base 2, what is taken off that, and the product with ln 2 round three times, a number of at most 1 + log2 E; the last sum is the one rounding of
the result. A score's gradient is p (g - sum p g), whose p sum up to 1: no part of its bound grows with the scores themselves, but with their differences alone."""
import math

import pytest

from tests.gpu_common import say
from tests.test_gpu_features import BF16, F32, TYPES, U, close, generator, normal
from tests.test_gpu_route import INF, exact_route, far_of, off

pytestmark = pytest.mark.gpu
torch = pytest.importorskip("torch")


@pytest.fixture(scope="module")
def ctx():
    from paper_2506_22668_amd import Context
    c = Context("cuda:0")
    yield c
    c.close()


def exact_gradient(p, ids, counts, dw, dloss, renorm):
    """(gradient, a bound of its parts' magnitudes) in 64 bits, from the probabilities."""
    experts, ids = p.shape[1], ids.long()
    g = torch.zeros_like(p)
    if dloss is not None:
        g += dloss.double() * experts * counts[:experts].double() / counts[:experts].sum().clamp(min=1) / counts[experts].clamp(min=1)
    size = g.abs()
    if dw is not None:
        held, at = (ids >= 0).double(), ids.clamp(min=0).t()
        dp, big = dw.double() * held, dw.double().abs() * held
        if renorm:
            w = p.gather(1, at).t() * held
            total = torch.where(w.sum(0) > 0, w.sum(0), 1.0)
            dp, big = held * (dp - (dp * w).sum(0) / total) / total, held * (big + (big * w).sum(0) / total) / total
        g, size = g.scatter_add(1, at, dp.t()), size.scatter_add(1, at, big.t())
    by = size + (p * size).sum(1, keepdim=True)
    return p * (g - (p * g).sum(1, keepdim=True)), p * by, 4 * 2.0 ** -150 * by


def check(ctx, g, x, k, renorm):
    rows, experts = x.shape
    ids, w, counts, loss, lse = ctx.route(x, k, renorm=renorm)
    ei, ew, ec, el, else_, p = exact_route(x, k, renorm)
    assert torch.equal(ids.long(), ei) and torch.equal(counts, ec)
    close(w, ew, 2 * (off(x) + (3 + k) * U) * ew + 3 * experts * 2.0 ** -150)
    close(loss, el, (off(x).max() + (rows + experts + 8) * U) * el)
    some = else_ > -INF
    assert torch.equal(lse > -INF, some)
    close(lse[some], else_[some], off(x)[some] + 3 * U * (1 + math.log2(experts)))
    dw, dloss = normal(g, k, rows), normal(g, 1) * 50
    for a, b in [(dw, dloss), (dw, None), (None, dloss)]:
        dx = ctx.route_backward(x, lse, ids, counts, dweights=a, dloss=b, renorm=renorm)
        e, size, least = exact_gradient(p, ids, counts, a, b, renorm)
        close(dx, e, (2 * experts + 64 + 8 * far_of(x) + 4 * k)[:, None] * U * size + least)


EXPERTS = [1, 2, 5, 8, 24, 64, 130, 515, 1024]


# (fp16 ends at 65,504)
@pytest.mark.parametrize("t, size", [(t, s) for t in TYPES for s in (0.0, 10.0, 300.0, 5000.0, 60000.0)] + [(t, s) for t in (F32, BF16) for s in (65500.0, 66000.0, 3e5, 1e7, 1e30)])
@pytest.mark.parametrize("sign", [1, -1])
def test_scores_far_from_zero(ctx, t, size, sign):
    """All scores of a row near one number of either sign; rows of different size beside each other."""
    say(f"route scores around {sign * size} {t}")
    for experts in EXPERTS:
        g = generator(experts)
        x = (sign * size + normal(g, 70, experts, scale=2.0)).to(t)
        x[torch.rand(70, experts, generator=g, device="cuda") < 0.1] = -INF
        x[::7] = normal(g, 10, experts).to(t)
        check(ctx, g, x, min(experts, 4), experts % 2 == 0)


@pytest.mark.parametrize("t, top", [(t, v) for t in TYPES for v in (0.0, 1e-40, 3e-5, 1.0, -3.7, 900.0, -60000.0)] + [(t, v) for t in (F32, BF16) for v in (66000.0, -1e5, 1e30)])
def test_scores_that_differ_in_their_last_bits(ctx, t, top):
    """Neighbouring numbers of the type, many of them equal."""
    say(f"route neighbours of {top} {t}")
    whole = torch.int32 if t == F32 else torch.int16
    for experts in EXPERTS:
        for k, steps in [(1, 3), (2, 2), (4, 7), (8, 40), (8, 1200)]:
            g = generator(experts + k)
            x = torch.full((50, experts), top, dtype=torch.float64, device="cuda").to(t)
            x = (x.view(whole) + torch.randint(0, steps, x.shape, generator=g, device="cuda").to(whole)).view(t)
            x = torch.where(torch.isfinite(x), x, torch.zeros_like(x))
            x[torch.rand(50, experts, generator=g, device="cuda") < 0.1] = -INF
            check(ctx, g, x, min(experts, k), k % 4 == 0)


@pytest.mark.parametrize("t", TYPES)
@pytest.mark.parametrize("experts", EXPERTS)
def test_gradient_where_a_mask_is_the_types_lowest_value(ctx, t, experts):
    """Rows masked throughout, in part, and not at all: a masked row's experts are alike."""
    say(f"route gradient of lowest values {t} experts={experts}")
    g = generator(experts)
    x = normal(g, 60, experts).to(t)
    low = torch.rand(60, experts, generator=g, device="cuda") < 0.5
    low[:20], low[50:] = True, False
    x[low] = torch.finfo(t).min
    ids, w, counts, loss, lse = ctx.route(x, 1)
    dw = normal(g, 1, 60)
    got = ctx.route_backward(x, lse, ids, counts, dweights=dw)
    p = exact_route(x, 1, False)[5]
    e, size, least = exact_gradient(p, ids, counts, dw, None, False)
    # (the differences that count are those of the rows' open scores; a score that far below has a probability of 0 on both sides)
    far = torch.where(low & ~low.all(1, keepdim=True), 0.0, x.double().amax(1, keepdim=True) - x.double()).amax(1)
    close(got, e, (2 * experts + 64 + 8 * far + 4)[:, None] * U * size + least)
