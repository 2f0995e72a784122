"""Operators on rows of features on the GPU against their formulas in 64 bits.

Tolerances. A result is rounded once to its type: half a step, eps / 2 of the type relative to the value (and half of the smallest
subnormal). Before that, fp32 arithmetic: a sum of n terms, whatever its order, is within n 2^-24 of the sum of the terms'
magnitudes, and the matrix cores are granted a second such share for what they cut off inside. Norms: mean, spread and result
together stay within 48 roundings (16 in a thread, 8 across threads, for each of the two sums, and the rest) of the largest value that
takes part."""
import numpy as np
import pytest

from oracle.philox import philox4x32_10_array
from tests.gpu_common import say

pytestmark = pytest.mark.gpu
torch = pytest.importorskip("torch")

F32, BF16, F16 = torch.float32, torch.bfloat16, torch.float16
TYPES = [F32, BF16, F16]
U = 2.0 ** -24
F64 = torch.float64


@pytest.fixture(scope="module")
def ctx():
    from paper_2506_22668_amd import Context
    c = Context("cuda:0")
    yield c
    c.close()


def rounding(t, exact):
    f = torch.finfo(t)
    return f.eps / 2 * exact.abs() + f.smallest_normal * f.eps / 2


def close(got, exact, before, t=None):
    """got within one rounding to its type of what `exact` is known to, `before`."""
    t = t or got.dtype
    assert torch.isfinite(got).all()
    far = (got.double() - exact).abs() - before - rounding(t, exact.abs() + before)
    assert far.max().item() <= 0, f"{far.max().item():.3e} too far, {int((far > 0).sum())} of {far.numel()} values"


def generator(seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    return g


def normal(g, *shape, t=F32, scale=1.0):
    return (torch.randn(*shape, generator=g, device="cuda") * scale).to(t)


def strided(a, pad, shift=0):
    """The rows of `a` with NaN between them, `shift` elements off the alignment of an allocation."""
    rows, cols = a.shape
    buf = torch.full((shift + rows * (cols + pad) + 8,), float("nan"), dtype=a.dtype, device="cuda")
    out = buf[shift:shift + rows * (cols + pad)].view(rows, cols + pad)[:, :cols]
    out.copy_(a)
    return out


# ---- layer norm ---------------------------------------------------------------------------------------------------------------

EPS = 1e-5


def norm_exact(x, w, b):
    x, w, b = x.double(), w.double(), b.double()
    mean = x.mean(1, keepdim=True)
    rstd = 1 / torch.sqrt((x - mean).square().mean(1, keepdim=True) + EPS)
    y = (x - mean) * rstd * w + b
    size = x.abs().amax(1, keepdim=True) * rstd * w.abs() + b.abs() + y.abs()
    return y, mean[:, 0], rstd[:, 0], size


WIDTHS = [1, 2, 7, 16, 31, 32, 33, 64, 100, 128, 129, 256, 515, 1000, 1024, 1025, 2047, 2048, 2049, 4095, 4096]


@pytest.mark.parametrize("t", TYPES)
@pytest.mark.parametrize("cols", WIDTHS)
def test_layer_norm_widths(ctx, t, cols):
    say(f"layer_norm {t} cols={cols}")
    g = generator(cols)
    for rows, pad, shift in [(1, 0, 0), (37, 3, 1)]:
        x = strided(normal(g, rows, cols, t=t) * 2 + 1, pad, shift)
        w, b = normal(g, cols), normal(g, cols)
        y, mean, rstd = ctx.layer_norm(x, w, b, want_stats=True)
        e, em, er, size = norm_exact(x, w, b)
        close(y, e, 48 * U * size)
        top = x.double().abs().amax(1)
        close(mean, em, 28 * U * top)
        close(rstd, er, 48 * U * (1 + top * er) * er)


@pytest.mark.parametrize("t", TYPES)
def test_layer_norm_many_rows_and_none(ctx, t):
    say(f"layer_norm many rows {t}")
    g = generator(5)
    x = normal(g, 70_001, 48, t=t)
    w, b = normal(g, 48), normal(g, 48)
    e, _, _, size = norm_exact(x, w, b)
    y = ctx.layer_norm(x, w, b)
    close(y, e, 48 * U * size)
    assert ctx.layer_norm(x[:0], w, b).shape == (0, 48)
    one, zero = torch.ones_like(w), torch.zeros_like(b)
    assert torch.equal(ctx.layer_norm(x), ctx.layer_norm(x, one, zero))
    assert torch.equal(ctx.layer_norm(x[:1].expand(9, 48), w, b), ctx.layer_norm(x[:1].repeat(9, 1), w, b))


@pytest.mark.parametrize("t", TYPES)
def test_layer_norm_of_a_transposed_view(ctx, t):
    say(f"layer_norm transposed {t}")
    g = generator(6)
    x = normal(g, 40, 23, t=t)
    w, b = normal(g, 23), normal(g, 23)
    assert torch.equal(ctx.layer_norm(x.t().contiguous().t(), w, b), ctx.layer_norm(x, w, b))


def test_layer_norm_of_constant_and_far_rows(ctx):
    """A constant row is its bias; rows far from zero keep the digits that their type has (two passes over the registers)."""
    say("layer_norm constant rows")
    w, b = torch.ones(300, device="cuda"), torch.full((300,), 0.25, device="cuda")
    assert torch.equal(ctx.layer_norm(torch.full((3, 300), 5.0, device="cuda"), w, b), torch.full((3, 300), 0.25, device="cuda"))
    g = generator(7)
    x = normal(g, 50, 300) + 1000.0
    e, _, _, size = norm_exact(x, w, b)
    close(ctx.layer_norm(x, w, b), e, 48 * U * size)


@pytest.mark.parametrize("t", TYPES)
def test_layer_norm_keeps_infinities_and_nan_to_their_rows(ctx, t):
    say(f"layer_norm non-finite {t}")
    g = generator(8)
    x = normal(g, 9, 70, t=t)
    want = ctx.layer_norm(x)
    x[2, 5], x[7, 69] = float("inf"), float("nan")
    y = ctx.layer_norm(x)
    assert torch.isnan(y[2]).all() and torch.isnan(y[7]).all()
    rest = [i for i in range(9) if i not in (2, 7)]
    assert torch.equal(y[rest], want[rest])


def norm_backward_exact(dy, x, mean, rstd, w):
    dy, x, w = dy.double(), x.double(), w.double()
    mean, rstd = mean.double()[:, None], rstd.double()[:, None]
    hat, g = (x - mean) * rstd, dy * w
    dx = rstd * (g - g.mean(1, keepdim=True) - hat * (g * hat).mean(1, keepdim=True))
    m = lambda v: v.abs().mean(1, keepdim=True)   # noqa: E731
    big = (x.abs() + mean.abs()) * rstd           # what xhat is a difference of
    size = rstd * (g.abs() + m(g) + big * m(g * hat) + hat.abs() * m(g * big))
    return dx, (dy * hat).sum(0), dy.sum(0), size, (dy.abs() * big).sum(0), dy.abs().sum(0)


@pytest.mark.parametrize("t", TYPES)
@pytest.mark.parametrize("cols", WIDTHS)
def test_layer_norm_backward_widths(ctx, t, cols):
    say(f"layer_norm_backward {t} cols={cols}")
    g = generator(cols + 1)
    for rows, pad, shift in [(1, 0, 0), (67, 5, 1)]:
        x, dy = strided(normal(g, rows, cols, t=t) * 2 + 1, pad, shift), strided(normal(g, rows, cols, t=t), pad + 1, shift)
        w = normal(g, cols)
        _, mean, rstd = ctx.layer_norm(x, w, want_stats=True)
        dx, dw, db = ctx.layer_norm_backward(dy, x, mean, rstd, w)
        ex, ew, eb, size, sw, sb = norm_backward_exact(dy, x, mean, rstd, w)
        close(dx, ex, 48 * U * size)
        close(dw, ew, (rows + 4) * U * sw)
        close(db, eb, rows * U * sb)


@pytest.mark.parametrize("t", TYPES)
@pytest.mark.parametrize("rows, cols", [(0, 12), (9_001, 40), (5_003, 1000), (4_100, 4096)])
def test_layer_norm_backward_rows(ctx, t, rows, cols):
    say(f"layer_norm_backward {t} {rows} x {cols}")
    g = generator(rows)
    x, dy, w = normal(g, rows, cols, t=t), normal(g, rows, cols, t=t), normal(g, cols)
    _, mean, rstd = ctx.layer_norm(x, want_stats=True)
    dx, dw, db = ctx.layer_norm_backward(dy, x, mean, rstd, w)
    if rows == 0:
        assert dx.shape == (0, cols) and not dw.any() and not db.any()
        return
    ex, ew, eb, size, sw, sb = norm_backward_exact(dy, x, mean, rstd, w)
    close(dx, ex, 48 * U * size)
    # rows are added up in a thread, a workgroup and across workgroups: far fewer roundings than rows meet any one of them
    close(dw, ew, 200 * U * sw)
    close(db, eb, 200 * U * sb)
    again = ctx.layer_norm_backward(dy, x, mean, rstd, w)
    assert all(torch.equal(a, b) for a, b in zip((dx, dw, db), again))


def test_layer_norm_backward_against_differences(ctx):
    say("layer_norm_backward differences")
    g = generator(9)
    x, w, b, c = normal(g, 6, 40), normal(g, 40), normal(g, 40), normal(g, 6, 40)
    _, mean, rstd = ctx.layer_norm(x, w, b, want_stats=True)
    got = ctx.layer_norm_backward(c, x, mean, rstd, w)
    h = 2.0 ** -7
    for which, grad in enumerate(got):
        v = normal(g, *grad.shape)
        p = [x, w, b]
        up, down = list(p), list(p)
        up[which], down[which] = p[which] + h * v, p[which] - h * v
        moved = (up[which].double() - down[which].double()) / 2   # (h v, as fp32 holds it)
        loss = lambda q: (ctx.layer_norm(*q).double() * c.double()).sum()   # noqa: E731
        plain = lambda q: (norm_exact(*q)[0] * c.double()).sum()   # noqa: E731
        slope = (loss(up) - loss(down)) / 2
        bent = (plain(up) - plain(down)) / 2                       # the same difference of the formula
        exact = norm_backward_exact(c, x, mean, rstd, w)[which]
        straight = (exact * moved).sum()
        noise = sum((48 * U * norm_exact(*q)[3] * c.double().abs() + rounding(F32, norm_exact(*q)[0]) * c.double().abs()).sum() for q in (up, down)) / 2
        assert abs(slope - (grad.double() * moved).sum()) <= abs(bent - straight) + noise + 200 * U * (exact.abs() * moved.abs()).sum()


# ---- dropout ------------------------------------------------------------------------------------------------------------------

def kept(rows, cols, p, seed, tag, first_row=0):
    calls = (cols + 7) // 8
    r = np.arange(first_row, first_row + rows, dtype=np.uint64)[:, None]
    c = np.arange(calls, dtype=np.uint64)[None, :]
    words = philox4x32_10_array(c + 0 * r, (r & np.uint64(0xFFFFFFFF)) + 0 * c, (r >> np.uint64(32)) + 0 * c, np.full((rows, calls), tag, np.uint64),
                                seed & 0xFFFFFFFF, seed >> 32)
    halves = np.stack([h for w in words for h in (w & np.uint64(0xFFFF), w >> np.uint64(16))], 2).reshape(rows, -1)[:, :cols]
    return torch.from_numpy((halves >= round(p * 65536)).astype(np.bool_)).cuda()


def drop_plain(x, keep, p, residual=None):
    """In fp32 as the kernel computes, one operation after the other: equal to the last bit."""
    t = round(p * 65536)
    v = torch.where(keep, x.float() * (65536.0 / (65536 - t) if t < 65536 else 0.0), 0.0)
    return (v if residual is None else residual.float() + v).to(x.dtype)


@pytest.mark.parametrize("t", TYPES)
@pytest.mark.parametrize("rows, cols, pad, shift", [(1, 1, 0, 0), (3, 7, 2, 1), (37, 129, 0, 0), (5, 8, 0, 1), (64, 1024, 8, 0), (1000, 515, 3, 1),
                                                    (2, 4097, 0, 0), (300_001, 16, 0, 0)])
def test_dropout_equals_its_definition(ctx, t, rows, cols, pad, shift):
    say(f"dropout {t} {rows} x {cols}")
    g = generator(rows + cols)
    x, r = strided(normal(g, rows, cols, t=t), pad, shift), strided(normal(g, rows, cols, t=t), pad + 1, shift)
    for p, seed, tag in [(0.1, 2 ** 61 + 12345, 1), (0.5, 7, 0xFFFFFFFF)]:
        keep = kept(rows, cols, p, seed, tag)
        assert torch.equal(ctx.dropout(x, p, seed, tag), drop_plain(x, keep, p))
        assert torch.equal(ctx.dropout(x, p, seed, tag, residual=r), drop_plain(x, keep, p, r))


@pytest.mark.parametrize("t", TYPES)
def test_dropout_ends_of_the_range(ctx, t):
    say(f"dropout ends {t}")
    x, r = normal(generator(1), 50, 50, t=t), normal(generator(2), 50, 50, t=t)
    assert torch.equal(ctx.dropout(x, 0.0, 3), x)
    assert torch.equal(ctx.dropout(x, 1.0, 3), torch.zeros_like(x))
    assert torch.equal(ctx.dropout(x, 1.0, 3, residual=r), r)
    assert ctx.dropout(x[:0], 0.3, 3).shape == (0, 50)
    assert torch.equal(ctx.dropout(x[:1].expand(50, 50), 0.3, 3), ctx.dropout(x[:1].repeat(50, 1), 0.3, 3))


@pytest.mark.parametrize("t", TYPES)
def test_dropped_infinities_and_nan_leave_nothing(ctx, t):
    say(f"dropout non-finite {t}")
    keep = kept(64, 96, 0.5, 11, 2)
    x = torch.where(keep, 1.0, float("nan")).to(t)
    x[::2] = torch.where(keep[::2], 1.0, float("inf")).to(t)
    y = ctx.dropout(x, 0.5, 11, 2)
    assert torch.equal(y, torch.where(keep, 2.0, 0.0).to(t))
    x = torch.where(keep, float("-inf"), 1.0).to(t)
    y = ctx.dropout(x, 0.5, 11, 2, residual=torch.ones_like(x))
    assert torch.equal(y, torch.where(keep, float("-inf"), 1.0).to(t))


def test_dropout_gradient_against_differences(ctx):
    """Linear in x: the difference is the gradient up to the roundings of its two forward passes."""
    say("dropout differences")
    g = generator(3)
    x, v, c = normal(g, 33, 65), normal(g, 33, 65), normal(g, 33, 65)
    dx = ctx.dropout(c, 0.3, 5, 9).double()
    up, down = (ctx.dropout(x + s * v, 0.3, 5, 9).double() * c.double() for s in (1.0, -1.0))
    moved = ((x + v).double() - (x - v).double()) / 2
    assert abs((up - down).sum() / 2 - (dx * moved).sum()) <= 4 * U * ((up.abs() + down.abs()).sum() + (dx * moved).abs().sum())


# ---- groups -------------------------------------------------------------------------------------------------------------------

@pytest.mark.parametrize("rows, groups", [(0, 3), (1, 1), (1, 256), (63, 2), (64, 64), (65, 5), (1010, 8), (4096, 7), (16_384, 3), (16_385, 1000),
                                          (20_001, 1), (100_003, 1024), (300_000, 64), (1_000_175, 64), (1_048_577, 255)])
def test_groups_equal_a_stable_sort(ctx, rows, groups):
    say(f"group_rows {rows} rows {groups} groups")
    rng = np.random.default_rng(rows + groups)
    ids = rng.integers(-1, groups + 1, rows).astype(np.int32)      # (some in no group, on both sides)
    if groups > 3:
        ids[ids == 2] = 1                                          # (one group empty, one large)
    if rows > 10:
        ids[3], ids[7] = np.iinfo(np.int32).min, np.iinfo(np.int32).max
    offsets, order = ctx.group_rows(torch.from_numpy(ids).cuda(), groups)
    key = np.where((ids >= 0) & (ids < groups), ids, groups)
    want = np.argsort(key, kind="stable")
    assert offsets.dtype == torch.int64 and order.dtype == torch.int32
    assert np.array_equal(order.cpu().numpy(), want)
    assert np.array_equal(offsets.cpu().numpy(), np.searchsorted(key[want], np.arange(groups + 1)))


@pytest.mark.parametrize("value", [-1, 0, 4])
def test_groups_where_all_rows_have_one(ctx, value):
    say(f"group_rows all {value}")
    for rows in (130, 40_000):
        offsets, order = ctx.group_rows(torch.full((rows,), value, dtype=torch.int32, device="cuda"), 5)
        assert torch.equal(order, torch.arange(rows, dtype=torch.int32, device="cuda"))
        assert offsets.tolist() == [0 if value < 0 or g <= value else rows for g in range(6)]


# ---- products by group ----------------------------------------------------------------------------------------------------------

def grouping(ctx, rng, rows, groups, order):
    """Ragged groups, one of them empty, some rows in none."""
    ids = np.minimum((groups + 1) * rng.random(rows) ** 1.5, groups).astype(np.int32) - (rng.random(rows) < 0.05)
    if groups >= 3:
        ids[ids == 1] = 0
    if not order:
        ids = np.sort(np.where(ids < 0, groups, ids)).astype(np.int32)
    offsets, perm = ctx.group_rows(torch.from_numpy(ids).cuda(), groups)
    key = torch.from_numpy(np.where((ids >= 0) & (ids < groups), ids, groups)).cuda()
    return offsets, (perm if order else None), key


def mm_exact(x, w, key, bias, relu):
    out = torch.zeros(x.shape[0], w.shape[2], dtype=F64, device="cuda")
    size = torch.zeros_like(out)
    for g in range(w.shape[0]):
        at = key == g
        y, s = x[at].double() @ w[g].double(), x[at].double().abs() @ w[g].double().abs()
        if bias is not None:
            y, s = y + bias[g].double(), s + bias[g].double().abs()
        out[at], size[at] = y.clamp(min=0) if relu else y, s
    return out, size


SHAPES = [(1, 1, 1, 1), (1, 16, 16, 3), (5, 40, 24, 4), (8, 256, 1000, 8), (33, 129, 65, 2), (64, 64, 128, 1), (70, 17, 300, 64),
          (200, 100, 36, 3), (300, 513, 130, 2), (1000, 128, 256, 5), (1111, 72, 520, 20), (2049, 264, 136, 3), (3001, 259, 515, 7),
          (5000, 512, 768, 4), (777, 1032, 40, 1)]


@pytest.mark.parametrize("t", TYPES)
@pytest.mark.parametrize("rows, inner, outer, groups", SHAPES)
def test_grouped_mm(ctx, t, rows, inner, outer, groups):
    say(f"grouped_mm {t} rows={rows} inner={inner} outer={outer} groups={groups}")
    rng, g = np.random.default_rng(rows), generator(inner)
    for order, pad, shift, bias, relu in [(True, 0, 0, True, True), (False, 3, 1, False, False)]:
        offsets, perm, key = grouping(ctx, rng, rows, groups, order)
        x, w = strided(normal(g, rows, inner, t=t), pad, shift), normal(g, groups, inner, outer, t=t, scale=inner ** -0.5)
        b = normal(g, groups, outer) if bias else None
        y = ctx.grouped_mm(x, w, offsets, order=perm, bias=b, relu=relu)
        e, size = mm_exact(x, w, key, b, relu)
        close(y, e, 2 * (inner + 2) * U * size)
        assert not y[key == groups].any()
        assert torch.equal(y, ctx.grouped_mm(x, w, offsets, order=perm, bias=b, relu=relu))


@pytest.mark.parametrize("t", TYPES)
@pytest.mark.parametrize("rows, inner, outer, groups", SHAPES)
def test_grouped_mm_backward(ctx, t, rows, inner, outer, groups):
    say(f"grouped_mm_backward {t} rows={rows} inner={inner} outer={outer} groups={groups}")
    rng, g = np.random.default_rng(rows + 1), generator(outer)
    for order, pad, shift, gated in [(True, 0, 0, True), (False, 3, 1, False)]:
        offsets, perm, key = grouping(ctx, rng, rows, groups, order)
        x, dy = normal(g, rows, inner, t=t), strided(normal(g, rows, outer, t=t), pad, shift)
        if gated:
            x = x.clamp(min=0)
        x = strided(x, pad + 1, shift)
        w = normal(g, groups, inner, outer, t=t, scale=inner ** -0.5)
        dx, dw, db = ctx.grouped_mm_backward(dy, x, w, offsets, order=perm, gate=x if gated else None)
        e, size = mm_exact(dy, w.transpose(1, 2), key, None, False)
        if gated:
            e, size = e.masked_fill(x <= 0, 0.0), size.masked_fill(x <= 0, 0.0)
        close(dx, e, 2 * (outer + 2) * U * size)
        assert not dx[key == groups].any()
        for k in range(groups):
            at = key == k
            xk, dk = x[at].double(), dy[at].double()
            n = int(at.sum())
            close(dw[k], xk.t() @ dk, 2 * n * U * (xk.abs().t() @ dk.abs()))
            close(db[k], dk.sum(0), 2 * n * U * dk.abs().sum(0))
        again = ctx.grouped_mm_backward(dy, x, w, offsets, order=perm, gate=x if gated else None)
        assert all(torch.equal(a, b) for a, b in zip((dx, dw, db), again))


# many tiles: workgroups go through several, the shortest contraction among them
@pytest.mark.parametrize("t", TYPES)
@pytest.mark.parametrize("rows, inner, outer, groups", [(70001, 16, 129, 2), (66001, 264, 136, 3), (40003, 131, 259, 7), (33000, 72, 520, 20)])
def test_grouped_mm_many_tiles(ctx, t, rows, inner, outer, groups):
    test_grouped_mm(ctx, t, rows, inner, outer, groups)
    test_grouped_mm_backward(ctx, t, rows, inner, outer, groups)


# few rows to a group: long contractions of few workgroups, and many workgroups
@pytest.mark.parametrize("t", TYPES)
@pytest.mark.parametrize("rows, inner, outer, groups", [(20, 2100, 136, 2), (50, 2101, 131, 2), (20, 136, 2100, 2), (50, 131, 2101, 2), (100, 72, 2056, 2),
                                                        (300, 520, 264, 40), (1000, 515, 257, 40), (2000, 520, 1024, 40)])
def test_grouped_mm_few_rows(ctx, t, rows, inner, outer, groups):
    test_grouped_mm(ctx, t, rows, inner, outer, groups)
    test_grouped_mm_backward(ctx, t, rows, inner, outer, groups)


# widths below a 16-byte piece, contractions that end right behind a step, matrices of less than 16 bytes
NARROW = [(3, 1, 1, 1), (1, 1, 2, 1), (2, 3, 1, 2), (40, 33, 3, 2), (40, 3, 33, 2), (90, 65, 1, 1), (90, 1, 65, 1), (700, 40, 5, 3), (700, 5, 40, 3),
          (300, 34, 9, 1), (200, 129, 130, 2), (1, 33, 7, 1), (33, 128, 7, 1), (600, 8, 8, 2), (600, 9, 15, 2)]


@pytest.mark.parametrize("t", TYPES)
@pytest.mark.parametrize("rows, inner, outer, groups", NARROW)
def test_grouped_mm_narrow(ctx, t, rows, inner, outer, groups):
    say(f"narrow {t} rows={rows} inner={inner} outer={outer} groups={groups}")
    test_grouped_mm(ctx, t, rows, inner, outer, groups)
    test_grouped_mm_backward(ctx, t, rows, inner, outer, groups)


@pytest.mark.parametrize("t", TYPES)
@pytest.mark.parametrize("rows", [1, 7, 100, 1000])
def test_grouped_mm_of_one_row_for_all(ctx, t, rows):
    """Rows that lie nowhere apart (an expanded row): their last piece is the buffer's last."""
    say(f"expanded {t} rows={rows}")
    g = generator(rows)
    for inner, outer in [(37, 45), (64, 264)]:
        x, dy, w = normal(g, 1, inner, t=t).expand(rows, inner), normal(g, 1, outer, t=t).expand(rows, outer), normal(g, 1, inner, outer, t=t)
        offsets = torch.tensor([0, rows], device="cuda")
        assert torch.equal(ctx.grouped_mm(x, w, offsets), ctx.grouped_mm(x.contiguous(), w, offsets))
        got, want = ctx.grouped_mm_backward(dy, x, w, offsets, gate=x), ctx.grouped_mm_backward(dy.contiguous(), x.contiguous(), w, offsets, gate=x.contiguous())
        assert all(torch.equal(a, b) for a, b in zip(got, want))


@pytest.mark.parametrize("t", TYPES)
def test_grouped_mm_without_rows(ctx, t):
    say(f"grouped_mm without rows {t}")
    w, offsets = normal(generator(1), 3, 40, 24, t=t), torch.zeros(4, dtype=torch.int64, device="cuda")
    x, dy = torch.empty(0, 40, dtype=t, device="cuda"), torch.empty(0, 24, dtype=t, device="cuda")
    assert ctx.grouped_mm(x, w, offsets).shape == (0, 24)
    dx, dw, db = ctx.grouped_mm_backward(dy, x, w, offsets)
    assert dx.shape == (0, 40) and not dw.any() and not db.any()
    # rows, but all of no group
    x, dy = normal(generator(2), 50, 40, t=t), normal(generator(3), 50, 24, t=t)
    assert not ctx.grouped_mm(x, w, offsets, bias=torch.ones(3, 24, device="cuda")).any()
    dx, dw, db = ctx.grouped_mm_backward(dy, x, w, offsets)
    assert not dx.any() and not dw.any() and not db.any()


@pytest.mark.parametrize("t", TYPES)
@pytest.mark.parametrize("rows", [40, 1500])
def test_grouped_mm_keeps_infinities_and_nan_to_their_group(ctx, t, rows):
    """Rows and weights of other groups, rows of no group and what lies between rows are not read into a sum."""
    say(f"grouped_mm non-finite {t} rows={rows}")
    rng, g = np.random.default_rng(rows), generator(4)
    inner, outer, groups = 75, 83, 4
    offsets, perm, key = grouping(ctx, rng, rows, groups, True)
    x, dy, w = normal(g, rows, inner, t=t), normal(g, rows, outer, t=t), normal(g, groups, inner, outer, t=t)
    bias = normal(g, groups, outer)
    clean = ctx.grouped_mm(x, w, offsets, order=perm, bias=bias, relu=True), *ctx.grouped_mm_backward(dy, x, w, offsets, order=perm)
    bad = (key == 2) | (key == groups)
    x[bad], dy[bad], w[2], bias[2] = float("nan"), float("inf"), float("nan"), float("nan")
    y = ctx.grouped_mm(x, w, offsets, order=perm, bias=bias, relu=True)
    dx, dw, db = ctx.grouped_mm_backward(dy, x, w, offsets, order=perm)
    ok, og = ~bad, [0, 1, 3]
    assert torch.equal(y[ok], clean[0][ok]) and torch.equal(dx[ok], clean[1][ok])
    assert torch.equal(dw[og], clean[2][og]) and torch.equal(db[og], clean[3][og])
    assert torch.isnan(y[key == 2]).all() and not y[key == groups].any()     # (a ReLU keeps a NaN)
    # a gate that is NaN lets nothing through
    gate = torch.full_like(x, float("nan"))
    assert not ctx.grouped_mm_backward(clean[0] * 0 + 1, normal(g, rows, inner, t=t), normal(g, groups, inner, outer, t=t), offsets,
                                       order=perm, gate=gate)[0].any()


@pytest.mark.parametrize("t", TYPES)
@pytest.mark.parametrize("rows", [40, 1500])
def test_orders_and_offsets_that_name_no_row_are_passed_over(ctx, t, rows):
    """The kernels' own bounds: the rows that are named properly come out right, nothing else is touched."""
    say(f"grouped_mm bad order {t} rows={rows}")
    g = generator(5)
    x, dy, w = normal(g, rows, 48, t=t), normal(g, rows, 56, t=t), normal(g, 2, 48, 56, t=t)
    offsets = torch.tensor([0, rows // 2, rows], device="cuda")
    order = torch.arange(rows, dtype=torch.int32, device="cuda")
    want, wdx, wdw, _ = ctx.grouped_mm(x, w, offsets), *ctx.grouped_mm_backward(dy, x, w, offsets)
    order[3], order[rows - 1] = -7, 2 ** 31 - 1
    y = ctx.grouped_mm(x, w, offsets, order=order)
    named = torch.ones(rows, dtype=torch.bool, device="cuda")
    named[3] = named[rows - 1] = False
    assert torch.equal(y[named], want[named])
    dx, dw, db = ctx.grouped_mm_backward(dy, x, w, offsets, order=order)
    assert torch.equal(dx[named], wdx[named])
    wild = torch.tensor([-2 ** 62, 2 ** 40, 2 ** 62], device="cuda")     # all rows in group 0, none behind
    assert torch.equal(ctx.grouped_mm(x, w, wild), ctx.grouped_mm(x, w, torch.tensor([0, rows, rows], device="cuda")))
    dw2 = ctx.grouped_mm_backward(dy, x, w, wild)[1]
    assert torch.equal(dw2, ctx.grouped_mm_backward(dy, x, w, torch.tensor([0, rows, rows], device="cuda"))[1])


def test_grouped_mm_gradients_against_differences(ctx):
    """The product is linear in each of x, w and bias: its difference is the gradient up to the roundings."""
    say("grouped_mm differences")
    rng, g = np.random.default_rng(1), generator(6)
    rows, inner, outer, groups = 90, 37, 29, 3
    offsets, perm, key = grouping(ctx, rng, rows, groups, True)
    x, w, b, c = normal(g, rows, inner), normal(g, groups, inner, outer), normal(g, groups, outer), normal(g, rows, outer)
    c[key == groups] = 0
    got = ctx.grouped_mm_backward(c, x, w, offsets, order=perm)
    for which, grad in enumerate(got):
        p, v = [x, w, b], normal(g, *grad.shape)
        if which == 0:
            v[key == groups] = 0
        up, down = list(p), list(p)
        up[which], down[which] = p[which] + v, p[which] - v
        moved = (up[which].double() - down[which].double()) / 2
        loss = [(ctx.grouped_mm(q[0], q[1], offsets, order=perm, bias=q[2]).double() * c.double()).sum() for q in (up, down)]
        noise = sum((2 * (inner + 3) * U * mm_exact(q[0], q[1], key, q[2], False)[1] * c.double().abs()).sum() for q in (up, down))
        assert abs((loss[0] - loss[1]) / 2 - (grad.double() * moved).sum()) <= noise + 2 * (rows + outer) * U * (grad.double() * moved).abs().sum()


# ---- the calls as a program makes them --------------------------------------------------------------------------------------------

def _all(ctx, s):
    y, mean, rstd = ctx.layer_norm(s["x"], s["w"], s["b"], want_stats=True)
    offsets, order = ctx.group_rows(s["ids"], 3)
    h = ctx.grouped_mm(y, s["m"], offsets, order=order, bias=s["mb"], relu=True)
    out = ctx.dropout(h, 0.2, 77, 1, residual=s["x"])
    dh = ctx.dropout(s["dy"], 0.2, 77, 1)
    dy, dm, dmb = ctx.grouped_mm_backward(dh, y, s["m"], offsets, order=order, gate=y)
    dx, dw, db = ctx.layer_norm_backward(dy, s["x"], mean, rstd, s["w"])
    return [y, mean, rstd, offsets, order, h, out, dm, dmb, dx, dw, db]


def _inputs(rows, seed):
    g = generator(seed)
    return dict(x=normal(g, rows, 136, t=BF16), w=normal(g, 136), b=normal(g, 136), m=normal(g, 3, 136, 136, t=BF16, scale=0.1),
                mb=normal(g, 3, 136), dy=normal(g, rows, 136, t=BF16), ids=torch.randint(-1, 3, (rows,), generator=g, device="cuda").int())


@pytest.mark.parametrize("rows", [50, 20_000])
def test_calls_on_another_stream_than_the_contexts(ctx, rows):
    say(f"streams rows={rows}")
    from paper_2506_22668_amd import Context
    s = _inputs(rows, 1)
    want = _all(ctx, s)
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    other = Context("cuda:0", stream=torch.cuda.Stream())
    for c in (ctx, other):
        with torch.cuda.stream(side):
            fresh = {k: torch.zeros_like(v) for k, v in s.items()}
            for k in s:                       # (inputs made on the side stream right before the calls)
                fresh[k].copy_(s[k])
            got = _all(c, fresh)
            got = [v.clone() for v in got]    # (and outputs used there right behind them)
        side.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(got, want))
    other.close()


@pytest.mark.parametrize("rows", [50, 20_000])
def test_calls_captured_into_a_graph(ctx, rows):
    say(f"graph rows={rows}")
    from paper_2506_22668_amd import Context
    stream = torch.cuda.Stream()
    mine = Context("cuda:0", stream=stream)
    s = _inputs(rows, 2)
    torch.cuda.synchronize()
    with torch.cuda.stream(stream):
        _all(mine, s)
    stream.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=stream):
        out = _all(mine, s)
    for seed in (3, 4, 5, 6):
        new = _inputs(rows, seed)
        for k in s:
            s[k].copy_(new[k])
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        want = _all(ctx, s)                  # (eager work between the replays)
        assert all(torch.equal(a, b) for a, b in zip(out, want)), seed
    mine.close()


def test_a_capture_of_another_stream_is_refused(ctx):
    say("graph of another stream")
    from paper_2506_22668_amd import DistShapError
    x = torch.ones(4, 8, device="cuda")
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        with pytest.raises(DistShapError):
            ctx.layer_norm(x)
        y = x + 1
    graph.replay()
    torch.cuda.synchronize()
    assert torch.equal(y, x + 1)


@pytest.mark.parametrize("t, element", [(F32, 0), (BF16, 1), (F16, 2)])
def test_outputs_with_rows_apart_and_in_place(ctx, t, element):
    """The C entries: what lies between the rows of an output stays as it was; an output over its input."""
    say(f"strided outputs {t}")
    lib, g = ctx.lib, generator(8)
    rows, cols, pad = 67, 53, 5
    x, w = normal(g, rows, cols, t=t), normal(g, cols)
    y, mean, rstd = ctx.layer_norm(x, w, want_stats=True)
    out = torch.full((rows, cols + pad), 3.0, dtype=t, device="cuda")
    assert lib.ds_layer_norm(ctx.h, element, rows, cols, x.data_ptr(), cols, w.data_ptr(), None, 1e-5, out.data_ptr(), cols + pad, None, None) == 0
    assert torch.equal(out[:, :cols], y) and (out[:, cols:] == 3).all()
    out.fill_(3.0)
    assert lib.ds_dropout(ctx.h, element, rows, cols, x.data_ptr(), cols, None, 0, 0.5, 4, 1, out.data_ptr(), cols + pad) == 0
    assert torch.equal(out[:, :cols], ctx.dropout(x, 0.5, 4, 1)) and (out[:, cols:] == 3).all()
    m = normal(g, 2, cols, 41, t=t)
    offsets = torch.tensor([0, 30, 60], device="cuda")
    out = torch.full((rows, 41 + pad), 3.0, dtype=t, device="cuda")
    assert lib.ds_grouped_mm(ctx.h, element, rows, cols, 41, 2, x.data_ptr(), cols, m.data_ptr(), offsets.data_ptr(), None, None, 0,
                             out.data_ptr(), 41 + pad) == 0
    assert torch.equal(out[:, :41], ctx.grouped_mm(x, m, offsets)) and (out[:, 41:] == 3).all()
    here = x.clone()
    assert lib.ds_layer_norm(ctx.h, element, rows, cols, here.data_ptr(), cols, w.data_ptr(), None, 1e-5, here.data_ptr(), cols, None, None) == 0
    assert torch.equal(here, y)
    here = x.clone()
    assert lib.ds_dropout(ctx.h, element, rows, cols, y.data_ptr(), cols, here.data_ptr(), cols, 0.5, 4, 1, here.data_ptr(), cols) == 0
    assert torch.equal(here, ctx.dropout(y, 0.5, 4, 1, residual=x))
    torch.cuda.synchronize()


def test_rows_behind_the_first_two_to_the_31_elements(ctx):
    """Offsets past 32 bits: the last rows of a buffer of more than 2^31 elements."""
    say("far rows")
    rows, cols = 540_001, 4096
    x = torch.zeros(rows, cols, dtype=BF16, device="cuda")
    x[-5:] = normal(generator(9), 5, cols, t=BF16)
    tail = ctx.layer_norm(x[-5:].clone())
    assert torch.equal(ctx.layer_norm(x)[-5:], tail)
    y = ctx.dropout(x, 0.25, 6, 3)
    assert torch.equal(y[-5:], drop_plain(x[-5:], kept(5, cols, 0.25, 6, 3, first_row=rows - 5), 0.25))
    del y
    w = normal(generator(10), 1, cols, 24, t=BF16, scale=0.02)
    offsets = torch.tensor([0, rows], device="cuda")
    out = ctx.grouped_mm(x, w, offsets)
    e, size = mm_exact(x[-5:], w, torch.zeros(5, dtype=torch.int64, device="cuda"), None, False)
    close(out[-5:], e, 2 * (cols + 2) * U * size)
