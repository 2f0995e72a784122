"""The calls on embeddings, routers and packed rows at their limits: the most rows they take, and rows in 8 bits that stand for the smallest and largest numbers of their type."""
import pytest

from tests.gpu_common import say
from tests.test_gpu_embed import gradient, shares
from tests.test_gpu_features import BF16, F16, F32, U, close, generator, normal

pytestmark = pytest.mark.gpu
torch = pytest.importorskip("torch")
MOST = 2 ** 30
PART = 2 ** 26


@pytest.fixture(scope="module")
def ctx():
    from paper_2506_22668_amd import Context
    c = Context("cuda:0")
    yield c
    c.close()


def test_the_most_rows_of_a_table(ctx):
    """2^30 rows of one column: each is the table's, or 0."""
    say("embed 2^30 rows")
    vocab = 1000
    ids = torch.randint(-1, vocab, (MOST,), generator=generator(1), device="cuda", dtype=torch.int32)
    table = normal(generator(2), vocab, 1)
    wide = torch.cat([table[:, 0], table.new_zeros(1)])
    y = ctx.embed(table, ids, dtype=BF16)
    assert y.shape == (MOST, 1)
    for first in range(0, MOST, PART):
        at = ids[first:first + PART].long()
        assert torch.equal(y[first:first + PART, 0], wide[at].to(BF16)), first   # (-1 is the zero behind the table)


@pytest.mark.parametrize("vocab", [1000, 3_000_000])
def test_the_most_rows_of_a_tables_gradient(ctx, vocab):
    """2^30 rows that are all the same: every sum is a whole number of at most 2^24 times a power of two, and exact."""
    say(f"embed_backward 2^30 rows vocab={vocab}")
    ids = torch.randint(-1, vocab, (MOST,), generator=generator(3), device="cuda", dtype=torch.int32)
    ids[5 * PART:5 * PART + 1_500_000] = vocab - 1           # (an id that reaches over many workgroups)
    of = torch.zeros(vocab + 1, dtype=torch.int64, device="cuda")
    for first in range(0, MOST, PART):
        of += torch.bincount(ids[first:first + PART].long() + 1, minlength=vocab + 1)
    dy = torch.tensor([[1.0, -0.5, 0.25]], device="cuda").to(BF16).expand(MOST, 3)
    got = ctx.embed_backward(dy, ids, vocab, dtype=F32)
    assert of[1:].max() <= 2 ** 24
    assert torch.equal(got, of[1:, None].float() * torch.tensor([[1.0, -0.5, 0.25]], device="cuda"))


@pytest.mark.parametrize("t, tt", [(F32, F32), (BF16, F32), (F16, F16)])
@pytest.mark.parametrize("how", ["one", "few", "uneven"])
@pytest.mark.parametrize("rows, vocab, cols", [(1024, 8, 40), (1025, 8, 40), (1024, 1, 130), (1025, 1, 130), (2048, 16, 64), (2049, 16, 64), (4096, 32, 9), (4000, 24, 72)])
def test_gradients_of_few_ids_at_the_borders_of_their_forms(ctx, t, tt, how, rows, vocab, cols):
    say(f"embed_backward {how} {t} rows={rows} vocab={vocab} cols={cols}")
    g = generator(rows)
    gradient(ctx, normal(g, rows, cols, t=t), shares(g, rows, vocab, how), vocab, 1.0, tt)


def test_the_most_rows_of_a_router(ctx):
    """2^30 rows of two experts, both of them each, and their gradient."""
    say("route 2^30 rows")
    x = torch.randn(MOST, 2, generator=generator(4), device="cuda", dtype=BF16)
    ids, w, counts, loss, lse = ctx.route(x, 2)
    assert counts.tolist() == [MOST, MOST, MOST]
    # (every expert has half of the choices, so the loss is 2 sum 1/2 p / N = 1; two terms a row, up to 2^12 rows in a thread, 2^9 threads)
    assert abs(loss.item() - 1) <= (2 + 16 + 2 ** 12 + 2 ** 9) * U
    dw = torch.ones(2, 1, device="cuda").expand(2, MOST).contiguous()
    dw[1] = -1.0
    dx = ctx.route_backward(x, lse, ids, counts, dweights=dw)
    for first in range(0, MOST, PART):
        at = slice(first, first + PART)
        v = x[at].float()
        high = (v[:, 1] > v[:, 0]).int()
        assert torch.equal(ids[0, at], high) and torch.equal(ids[1, at], 1 - high), first
        far = (v[:, 0] - v[:, 1]).abs()
        p = torch.sigmoid(far)
        # (torch's fp32 and the kernel's, each within the roundings of tests/test_gpu_route.py)
        off = 2 * (2 + 16 + 2 * far + 5) * U
        assert ((w[0, at] - p).abs() <= 2 * off * p).all() and ((w[1, at] - (1 - p)).abs() <= 2 * off * p).all(), first
        assert ((lse[at] - (v.amax(1) - torch.log(p))).abs() <= 2 * off * (1 + v.abs().amax(1))).all(), first
        # dw of 1 for the higher and -1 for the other: 2 p (1 - p), and its negative; one rounding of the result to bf16
        g = 2 * p * (1 - p)
        e = torch.where(high[:, None] == torch.arange(2, device="cuda"), g[:, None], -g[:, None])
        assert ((dx[at].float() - e).abs() <= 2.0 ** -8 * e.abs() + 2 * off[:, None] * 4).all(), first


# ---- rows in 8 bits at the ends of the types -------------------------------------------------------------------------------------

# (powers of two that the rows and their gradients are multiplied by: rows between the smallest subnormals and a little above the smallest normal
# number, at the type's largest, and both beside each other)
ENDS = [(F16, -18, 8), (F16, -14, 6), (F16, 11, -8), (BF16, -128, 60), (BF16, -122, 60), (BF16, 120, -60), (F32, -110, 60), (F32, 120, -60)]


@pytest.mark.parametrize("t, of_x, of_dy", ENDS)
@pytest.mark.parametrize("rows, inner, outer", [(40, 72, 64), (9, 33, 25), (3000, 256, 128), (3001, 259, 131), (40_000, 512, 256)])
def test_gradients_from_codes_of_the_smallest_and_largest_numbers(ctx, t, of_x, of_dy, rows, inner, outer):
    """The weights' gradient is that of the rows that the codes stand for, subnormal numbers among them."""
    say(f"packed gradients of 2^{of_x} {t} rows={rows} inner={inner}")
    g = generator(rows)
    x = (normal(g, rows, inner).clamp(-3, 3).double() * 2.0 ** of_x).to(t)
    x[::3] = (x[::3].double() * 2.0 ** (-6 if of_x < 0 else -20)).to(t)
    dy, w = (normal(g, rows, outer).double() * 2.0 ** of_dy).to(t), normal(g, 2, inner, outer, t=t)
    p = ctx.pack_rows(x)
    held = ctx.unpack_rows(p, t)
    assert torch.isfinite(held).all() and torch.equal(held == 0, x == 0)
    offsets = torch.tensor([0, rows // 3, rows], device="cuda")
    dx, dw, db = ctx.grouped_mm_backward(dy, p, w, offsets, gate=p)
    for k, at in enumerate((slice(0, rows // 3), slice(rows // 3, rows))):
        xk, dk = held[at].double(), dy[at].double()
        n = xk.shape[0]
        # (a sum's terms are at or above 2^-149 in fp32, or lost: n halves of that at the most)
        close(dw[k], xk.t() @ dk, 2 * n * U * (xk.abs().t() @ dk.abs()) + n * 2.0 ** -149)
    open_ = ctx.grouped_mm_backward(dy, p, w, offsets)[0]
    assert torch.equal(dx, torch.where(x > 0, open_, torch.zeros_like(open_)))
