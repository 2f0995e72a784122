"""Rows of a table by id and the table's gradient on the GPU against their formulas.

Tolerances. A looked-up row is one product, in fp32 and then rounded to its type, or rounded to its type alone where one instruction does both (fp16: 1.2890625
times the fp32 number next to 22.6 is 29.13281299, above the middle 29.1328125 of two fp16 numbers, and 29.140625 if it is rounded once; fp32 has the middle itself next to
it, which then goes to the even 29.125): within 2^-24 of the product and one rounding, and equal bit by bit where the scale is a power of two. A row of
the gradient is a sum of n terms in fp32, in whatever order, within n 2^-24 of the sum of the terms' magnitudes, times the scale (one more
rounding), rounded once to the table's type."""
import pytest

from tests.gpu_common import say
from tests.test_gpu_features import BF16, F16, F32, TYPES, U, close, generator, normal, strided

pytestmark = pytest.mark.gpu
torch = pytest.importorskip("torch")

PAIRS = [(F32, F32), (BF16, BF16), (F16, F16), (BF16, F32), (F16, F32)]   # of the rows, of the table


@pytest.fixture(scope="module")
def ctx():
    from paper_2506_22668_amd import Context
    c = Context("cuda:0")
    yield c
    c.close()


def looked_up(table, ids, scale, t):
    there = (ids >= 0) & (ids < table.shape[0])
    rows = table[ids.clamp(0, table.shape[0] - 1).long()].float() * torch.tensor(scale, device="cuda")
    return torch.where(there[:, None], rows, 0.0).to(t)


def some_ids(g, rows, vocab):
    """Ids of all of a table, some of them -1, one behind its end, the largest and the lowest there are."""
    ids = torch.randint(-1, vocab + 1, (rows,), generator=g, device="cuda").int()
    if rows > 4:
        ids[1], ids[3] = 2 ** 31 - 1, -2 ** 31
    return ids


WIDTHS = [1, 2, 3, 4, 5, 7, 8, 9, 15, 16, 31, 33, 64, 100, 129, 515, 1024, 4097]


@pytest.mark.parametrize("t, tt", PAIRS)
@pytest.mark.parametrize("cols", WIDTHS)
def test_rows_of_a_table(ctx, t, tt, cols):
    say(f"embed {t} of {tt} cols={cols}")
    g = generator(cols)
    for rows, vocab, scale, pad, shift in [(1, 1, 1.0, 0, 0), (37, 11, 22.6, 3, 1), (3001, 700, -0.5, 0, 0)]:
        table, ids = strided(normal(g, vocab, cols, t=tt), pad, shift), some_ids(g, rows, vocab)
        y = ctx.embed(table, ids, scale=scale, dtype=t)
        exact = torch.where(((ids >= 0) & (ids < vocab))[:, None], table[ids.clamp(0, vocab - 1).long()].double() * torch.tensor(scale).double().item(), 0.0)
        assert y.dtype == t
        close(y, exact, U * exact.abs())
        if scale != 22.6:
            assert torch.equal(y, looked_up(table, ids, scale, t))


@pytest.mark.parametrize("t, tt", PAIRS)
def test_rows_of_a_table_beyond_the_ordinary(ctx, t, tt):
    say(f"embed no rows, one row for all, transposed {t} of {tt}")
    g = generator(3)
    table, ids = normal(g, 50, 40, t=tt), some_ids(g, 90, 50)
    want = looked_up(table, ids, 1.0, t)
    assert ctx.embed(table, ids[:0], dtype=t).shape == (0, 40)
    assert torch.equal(ctx.embed(table.t().contiguous().t(), ids, dtype=t), want)
    assert torch.equal(ctx.embed(table[:1].expand(50, 40), ids, dtype=t), looked_up(table[:1].repeat(50, 1), ids, 1.0, t))
    assert torch.equal(ctx.embed(table, ids.repeat_interleave(2)[::2], dtype=t), want)
    # what is not looked up is not seen: rows of no id are zeros though the table holds nothing finite
    table[0], table[49, 3] = float("nan"), float("inf")
    y = ctx.embed(table, torch.tensor([-1, 0, 49, 50, 7], device="cuda").int(), dtype=t)
    assert not y[0].any() and not y[3].any() and torch.isnan(y[1]).all() and torch.isinf(y[2, 3]) and torch.isfinite(y[4]).all()
    assert y[2].isinf().sum() == 1


def gradient(ctx, dy, ids, vocab, scale, tt):
    """The call, held to the formula in 64 bits."""
    got = ctx.embed_backward(dy, ids, vocab, scale=scale, dtype=tt)
    assert got.dtype == tt and got.shape == (vocab, dy.shape[1])
    known = ((ids >= 0) & (ids < vocab)).nonzero()[:, 0]
    at, rows = ids[known].long(), dy[known].double().cpu()   # (many rows of one id: the CPU adds them up in order, without atomics)
    scale = torch.tensor(scale).double().item()   # (fp32)
    zeros = torch.zeros(vocab, dy.shape[1], dtype=torch.float64)
    exact = zeros.clone().index_add_(0, at.cpu(), rows).cuda() * scale
    size = zeros.index_add_(0, at.cpu(), rows.abs()).cuda() * abs(scale)
    n = torch.bincount(at, minlength=vocab)[:, None]
    close(got, exact, (n + 1) * U * size)
    assert not got[n[:, 0] == 0].any()
    assert torch.equal(got, ctx.embed_backward(dy, ids, vocab, scale=scale, dtype=tt))
    return got


@pytest.mark.parametrize("t, tt", PAIRS)
@pytest.mark.parametrize("cols", WIDTHS)
def test_gradient_widths(ctx, t, tt, cols):
    say(f"embed_backward {t} of {tt} cols={cols}")
    g = generator(cols + 1)
    for rows, vocab, scale, pad, shift in [(1, 1, 1.0, 0, 0), (37, 11, 22.625, 3, 1), (3001, 700, -0.5, 0, 0)]:
        gradient(ctx, strided(normal(g, rows, cols, t=t), pad, shift), some_ids(g, rows, vocab), vocab, scale, tt)


def shares(g, rows, vocab, how):
    if how == "one":
        return torch.full((rows,), vocab // 2, dtype=torch.int32, device="cuda")
    if how == "none":
        return torch.full((rows,), -1, dtype=torch.int32, device="cuda")
    if how == "once":
        return torch.randperm(vocab, generator=g, device="cuda")[:rows].int()
    if how == "sorted":
        return torch.sort(torch.randint(0, vocab, (rows,), generator=g, device="cuda"))[0].int()
    if how == "few":   # (half of the rows have one id)
        ids = torch.randint(0, vocab, (rows,), generator=g, device="cuda")
        return torch.where(torch.rand(rows, generator=g, device="cuda") < 0.5, vocab - 1, ids).int()
    return (torch.rand(rows, generator=g, device="cuda").pow(6) * vocab).int().clamp(max=vocab - 1)   # "uneven"


# one digit, two and three; one workgroup and several that sort; stretches that end inside an id's rows
@pytest.mark.parametrize("t, tt", [(F32, F32), (BF16, F32), (F16, F16)])
@pytest.mark.parametrize("how", ["one", "none", "once", "sorted", "few", "uneven"])
@pytest.mark.parametrize("rows, vocab, cols", [(2, 3, 8), (16, 1023, 24), (17, 1024, 8), (255, 300, 40), (1000, 1000, 16), (2049, 5000, 72), (8191, 1_100_000, 4),
                                               (8192, 8192, 16), (8193, 70_000, 9), (4096, 511, 24), (4097, 511, 24), (8192, 511, 8), (8192, 512, 131), (6000, 400, 16), (20_011, 40_000, 33), (70_000, 1023, 64), (262_145, 300_000, 12)])
def test_gradient_of_ids_in_any_shares(ctx, t, tt, how, rows, vocab, cols):
    say(f"embed_backward {how} {t} rows={rows} vocab={vocab} cols={cols}")
    g = generator(rows)
    if how == "once" and rows > vocab:
        rows = vocab
    gradient(ctx, normal(g, rows, cols, t=t), shares(g, rows, vocab, how), vocab, 1.0, tt)


@pytest.mark.parametrize("t, tt", PAIRS)
def test_gradient_beyond_the_ordinary(ctx, t, tt):
    say(f"embed_backward no rows, one row for all, transposed, non-finite {t} of {tt}")
    g = generator(4)
    dy, ids = normal(g, 300, 40, t=t), some_ids(g, 300, 20)
    want = gradient(ctx, dy, ids, 20, 1.0, tt)
    assert not ctx.embed_backward(dy[:0], ids[:0], 20, dtype=tt).any()
    assert torch.equal(ctx.embed_backward(dy.t().contiguous().t(), ids, 20, dtype=tt), want)
    gradient(ctx, dy[:1].expand(300, 40), ids, 20, 1.0, tt)
    dy[5, 3], dy[7, 8] = float("inf"), float("nan")   # stay with their ids and columns
    got = ctx.embed_backward(dy, ids, 20, dtype=tt)
    for r, c in [(5, 3), (7, 8)]:
        if 0 <= ids[r] < 20:
            assert not torch.isfinite(got[ids[r].item(), c])
            got[ids[r].item(), c] = want[ids[r].item(), c]
    assert torch.equal(got, want)


def test_gradient_against_differences(ctx):
    """The lookup is linear in the table: its difference is the gradient up to the roundings."""
    say("embed differences")
    g = generator(5)
    table, move, ids = normal(g, 90, 33), normal(g, 90, 33), some_ids(g, 400, 90)
    c = normal(g, 400, 33)
    grad = ctx.embed_backward(c, ids, 90, scale=3.0).double()
    up, down = table + move, table - move
    moved = (up.double() - down.double()) / 2
    a, b = ctx.embed(up, ids, scale=3.0).double(), ctx.embed(down, ids, scale=3.0).double()
    noise = U * ((a.abs() + b.abs()) * c.double().abs()).sum() + 401 * U * (ctx.embed_backward(c.abs(), ids, 90, scale=3.0).double() * moved.abs()).sum()
    assert abs(((a - b) / 2 * c.double()).sum() - (grad * moved).sum()) <= noise


@pytest.mark.parametrize("t, tt", PAIRS)
def test_outputs_with_rows_apart(ctx, t, tt):
    """The C entries: what lies between the rows of an output, and behind a workspace, stays as it was."""
    say(f"embed strided outputs {t} of {tt}")
    import ctypes as C
    lib, g = ctx.lib, generator(8)
    for rows, vocab, cols, pad in [(67, 41, 53, 5), (9000, 3000, 20, 3)]:
        table, ids, dy = normal(g, vocab, cols, t=tt), some_ids(g, rows, vocab), normal(g, rows, cols, t=t)
        a, b = ctx._elements[t], ctx._elements[tt]
        out = torch.full((rows, cols + pad), 3.0, dtype=t, device="cuda")
        assert lib.ds_embed(ctx.h, a, b, rows, cols, vocab, table.data_ptr(), cols, ids.data_ptr(), 1.0, out.data_ptr(), cols + pad) == 0
        assert torch.equal(out[:, :cols], ctx.embed(table, ids, dtype=t)) and (out[:, cols:] == 3).all()
        need = C.c_int64()
        assert lib.ds_embed_backward_workspace(rows, cols, vocab, C.byref(need)) == 0
        ws = torch.full((need.value + 64,), 77, dtype=torch.uint8, device="cuda")
        out = torch.full((vocab, cols + pad), 3.0, dtype=tt, device="cuda")
        assert lib.ds_embed_backward(ctx.h, a, b, rows, cols, vocab, dy.data_ptr(), cols, ids.data_ptr(), 1.0, out.data_ptr(), cols + pad, ws.data_ptr(),
                                     need.value) == 0
        assert torch.equal(out[:, :cols], ctx.embed_backward(dy, ids, vocab, dtype=tt)) and (out[:, cols:] == 3).all() and (ws[need.value:] == 77).all()
    torch.cuda.synchronize()


def test_rows_behind_the_first_two_to_the_31_elements(ctx):
    say("embed far rows")
    vocab, cols = 540_001, 4096
    table = torch.zeros(vocab, cols, dtype=BF16, device="cuda")
    table[-5:] = normal(generator(9), 5, cols, t=BF16)
    ids = torch.tensor([vocab - 1, 0, vocab - 5, vocab], device="cuda").int()
    assert torch.equal(ctx.embed(table, ids), looked_up(table, ids, 1.0, BF16))
    far = torch.arange(vocab, device="cuda").int()
    far[:-5] = -1
    y = ctx.embed(table, far)                       # rows of the output past 2^31 elements
    assert torch.equal(y[-5:], table[-5:]) and not y[:-5].any()
    grad = ctx.embed_backward(y, far, vocab)        # rows of dy and of the table's gradient
    assert torch.equal(grad[-5:], table[-5:]) and not grad[:-5].any()
