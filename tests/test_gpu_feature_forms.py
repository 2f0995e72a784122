"""Forms of the operators on rows of features that the sizes alone do not reach: operands that lie as the direct loads of the tiles need
them, more groups than a wave or a workgroup looks at in one go, orders with holes, outputs over inputs, and buffers of more than 2^31
elements backwards. Tolerances are those of test_gpu_features.py."""
import numpy as np
import pytest

from tests import test_gpu_features as features
from tests.gpu_common import say
from tests.test_gpu_features import (BF16, EPS, F16, F32, TYPES, U, close, ctx, generator, grouping, mm_exact, norm_backward_exact,   # noqa: F401
                                     normal, strided)

pytestmark = pytest.mark.gpu
torch = pytest.importorskip("torch")


def check_backward(ctx, dy, x, w, offsets, perm, key, gate):   # noqa: F811
    """Both gradients against 64 bits, and the same bits again."""
    got = dx, dw, db = ctx.grouped_mm_backward(dy, x, w, offsets, order=perm, gate=gate)
    e, size = mm_exact(dy, w.transpose(1, 2), key, None, False)
    if gate is not None:
        e, size = e.masked_fill(~(gate > 0), 0.0), size.masked_fill(~(gate > 0), 0.0)
    close(dx, e, 2 * (w.shape[2] + 2) * U * size)
    assert not dx[key >= w.shape[0]].any()
    for k in range(w.shape[0]):
        at = key == k
        xk, dk, n = x[at].double(), dy[at].double(), int(at.sum())
        close(dw[k], xk.t() @ dk, 2 * n * U * (xk.abs().t() @ dk.abs()))
        close(db[k], dk.sum(0), 2 * n * U * dk.abs().sum(0))
    again = ctx.grouped_mm_backward(dy, x, w, offsets, order=perm, gate=gate)
    assert all(torch.equal(a, b) for a, b in zip(got, again))


# x and dy on 16 bytes, their rows whole pieces of 16 bytes apart: the gradient of the weights loads them into LDS directly. apart: 0 or a piece.
@pytest.mark.parametrize("t", TYPES)
@pytest.mark.parametrize("rows, inner, outer, groups", [(5000, 512, 768, 4), (3001, 256, 512, 7), (2049, 264, 136, 3), (1500, 1032, 40, 1),
                                                        (40003, 136, 256, 7), (33000, 72, 520, 20), (66001, 264, 136, 3)])
@pytest.mark.parametrize("apart", [0, 8])
def test_gradients_of_aligned_rows(ctx, t, rows, inner, outer, groups, apart):   # noqa: F811
    say(f"aligned {t} rows={rows} inner={inner} outer={outer} groups={groups} apart={apart}")
    rng, g = np.random.default_rng(rows), generator(inner + apart)
    for order in (True, False):
        offsets, perm, key = grouping(ctx, rng, rows, groups, order)
        x, dy = strided(normal(g, rows, inner, t=t), apart), strided(normal(g, rows, outer, t=t), apart)
        assert x.data_ptr() % 16 == 0 and dy.data_ptr() % 16 == 0
        w = normal(g, groups, inner, outer, t=t, scale=inner ** -0.5)
        check_backward(ctx, dy, x, w, offsets, perm, key, x if order else None)


# the tiles that test_gpu_features.py does not come to: fp32 of 128 rows, rows of whole pieces and odd ones, and dx of 256; 17 to 32 rows to a group
# whose dx has many workgroups (tests/test_grouped_forms.py says which form a shape takes)
@pytest.mark.parametrize("t", TYPES)
@pytest.mark.parametrize("rows, inner, outer, groups", [(6000, 131, 515, 2), (6000, 515, 130, 2), (3000, 1024, 64, 2), (4000, 2048, 128, 1), (40_003, 388, 133, 3),
                                                        (600, 1032, 1032, 20)])
def test_products_of_further_forms(ctx, t, rows, inner, outer, groups):   # noqa: F811
    features.test_grouped_mm(ctx, t, rows, inner, outer, groups)
    features.test_grouped_mm_backward(ctx, t, rows, inner, outer, groups)


def many_groups(ctx, seed, rows, groups, order):   # noqa: F811
    """Ragged groups of which a third is empty, the first, the last and those next to multiples of 64 and 256 not among them; some rows in none."""
    rng = np.random.default_rng(seed)
    held = np.array([k for k in range(groups) if k % 3 != 1 or k % 64 in (0, 1, 63) or k == groups - 1])
    ids = held[np.minimum(len(held) * rng.random(rows) ** 1.3, len(held) - 1).astype(np.int64)].astype(np.int32)
    edge = [k for k in (0, 63, 64, 65, 255, 256, 257, 511, 512, 600, groups - 1) if k < groups and k in held]
    ids[:2 * len(edge)] = edge * 2
    ids[rng.random(rows) < 0.03] = -1
    if not order:
        ids = np.sort(np.where(ids < 0, groups, ids)).astype(np.int32)
    offsets, perm = ctx.group_rows(torch.from_numpy(ids).cuda(), groups)
    return offsets, (perm if order else None), torch.from_numpy(np.where(ids < 0, groups, ids)).cuda()


# the first four: few rows to a group (rows that the waves share, and not); then tiles of rows, of weights, or both
@pytest.mark.parametrize("t", TYPES)
@pytest.mark.parametrize("rows, inner, outer, groups", [(900, 24, 40, 65), (6000, 40, 72, 130), (2000, 24, 16, 600), (9000, 16, 24, 1024),
                                                        (30_000, 64, 264, 65), (60_000, 128, 136, 257), (150_000, 72, 256, 600),
                                                        (200_000, 256, 64, 1024), (150_000, 131, 67, 513)])
def test_products_of_many_groups(ctx, t, rows, inner, outer, groups):   # noqa: F811
    say(f"many groups {t} rows={rows} inner={inner} outer={outer} groups={groups}")
    g = generator(groups)
    for order in (True, False):
        offsets, perm, key = many_groups(ctx, groups, rows, groups, order)
        x, dy = normal(g, rows, inner, t=t), normal(g, rows, outer, t=t)
        w, bias = normal(g, groups, inner, outer, t=t, scale=inner ** -0.5), normal(g, groups, outer)
        y = ctx.grouped_mm(x, w, offsets, order=perm, bias=bias, relu=order)
        e, size = mm_exact(x, w, key, bias, order)
        close(y, e, 2 * (inner + 2) * U * size)
        assert not y[key == groups].any()
        check_backward(ctx, dy, x, w, offsets, perm, key, x if order else None)


@pytest.mark.parametrize("t", TYPES)
@pytest.mark.parametrize("rows, inner, outer", [(40, 48, 56), (100, 48, 56), (1500, 48, 56), (6000, 264, 256)])
def test_orders_with_holes_add_no_other_row(ctx, t, rows, inner, outer):   # noqa: F811
    """Positions of the order that name no row leave nothing in a gradient; row 0, which a kernel would read in their place, is large."""
    say(f"order with holes {t} rows={rows} {inner} x {outer}")
    g = generator(rows)
    x, dy, w = normal(g, rows, inner, t=t), normal(g, rows, outer, t=t), normal(g, 2, inner, outer, t=t, scale=inner ** -0.5)
    x[0], dy[0] = 100.0, 50.0
    offsets = torch.tensor([0, rows // 2, rows], device="cuda")
    order, key = torch.arange(rows, dtype=torch.int32, device="cuda"), torch.zeros(rows, dtype=torch.int64, device="cuda")
    key[rows // 2:] = 1
    holes = torch.tensor([3, rows // 2 - 1, rows // 2, rows - 6, rows - 1], device="cuda")
    order[holes] = torch.tensor([-7, 2 ** 31 - 1, -2 ** 31, rows, -1], dtype=torch.int32, device="cuda")
    named = torch.ones(rows, dtype=torch.bool, device="cuda")
    named[holes] = False
    y = ctx.grouped_mm(x, w, offsets, order=order)
    e, size = mm_exact(x, w, key, None, False)
    close(y[named], e[named], (2 * (inner + 2) * U * size)[named])
    dx, dw, db = ctx.grouped_mm_backward(dy, x, w, offsets, order=order)
    e, size = mm_exact(dy, w.transpose(1, 2), key, None, False)
    close(dx[named], e[named], (2 * (outer + 2) * U * size)[named])
    for k in range(2):
        at = named & (key == k)
        xk, dk, n = x[at].double(), dy[at].double(), int(at.sum())
        close(dw[k], xk.t() @ dk, 2 * n * U * (xk.abs().t() @ dk.abs()))
        close(db[k], dk.sum(0), 2 * n * U * dk.abs().sum(0))


@pytest.mark.parametrize("t, element", [(F32, 0), (BF16, 1), (F16, 2)])
@pytest.mark.parametrize("rows, cols, pad", [(67, 53, 5), (3, 4096, 0), (2000, 515, 0), (700, 2049, 3)])
def test_norm_gradient_over_its_inputs(ctx, t, element, rows, cols, pad):   # noqa: F811
    """dx in the buffer of dy, and in that of x, with equal strides."""
    say(f"layer_norm_backward in place {t} {rows} x {cols}")
    g = generator(cols)
    x, dy, w = strided(normal(g, rows, cols, t=t), pad), strided(normal(g, rows, cols, t=t), pad), normal(g, cols)
    _, mean, rstd = ctx.layer_norm(x, w, want_stats=True)
    want = ctx.layer_norm_backward(dy, x, mean, rstd, w)
    ex, ew, eb, size, sw, sb = norm_backward_exact(dy, x, mean, rstd, w)
    close(want[0], ex, 48 * U * size)
    ws, ptr, n = ctx._workspace(ctx.lib.ds_layer_norm_backward_workspace, rows, cols)
    for over in ("dy", "x"):
        a, b = strided(dy, pad), strided(x, pad)
        dx = a if over == "dy" else b
        dw, db = torch.full((2, cols), float("nan"), device="cuda")
        assert ctx.lib.ds_layer_norm_backward(ctx.h, element, rows, cols, a.data_ptr(), cols + pad, b.data_ptr(), cols + pad, mean.data_ptr(),
                                              rstd.data_ptr(), w.data_ptr(), dx.data_ptr(), cols + pad, dw.data_ptr(), db.data_ptr(), ptr, n) == 0
        assert torch.equal(dx, want[0]) and torch.equal(dw, want[1]) and torch.equal(db, want[2])
    torch.cuda.synchronize()


def test_gradients_of_rows_behind_the_first_two_to_the_31_elements(ctx):   # noqa: F811
    """Offsets past 32 bits backwards: only the first and the last rows of a buffer of more than 2^31 elements are not zero."""
    say("far rows backward")
    rows, cols, outer = 540_001, 4096, 24
    ends = torch.tensor([0, 1, 2, rows - 5, rows - 4, rows - 3, rows - 2, rows - 1], device="cuda")
    g = generator(11)
    x = torch.zeros(rows, cols, dtype=BF16, device="cuda")
    x[ends] = normal(g, 8, cols, t=BF16)
    mean, rstd = torch.zeros(rows, device="cuda"), torch.ones(rows, device="cuda")
    e = x[ends].double()
    mean[ends], rstd[ends] = e.mean(1).float(), (1 / torch.sqrt(e.var(1, unbiased=False) + EPS)).float()
    near, w = normal(g, 8, cols, t=BF16), normal(g, cols)
    dy = torch.zeros_like(x)
    dy[ends] = near
    dx, dw, db = ctx.layer_norm_backward(dy, x, mean, rstd, w)
    ex, ew, eb, size, sw, sb = norm_backward_exact(near, x[ends], mean[ends], rstd[ends], w)
    close(dx[ends], ex, 48 * U * size)
    close(dw, ew, 48 * U * sw)
    close(db, eb, 48 * U * sb)
    assert not dx[1000:rows - 1000].any()
    del dy, dx
    m = normal(g, 1, cols, outer, t=BF16, scale=cols ** -0.5)
    dy = torch.zeros(rows, outer, dtype=BF16, device="cuda")
    dy[ends] = normal(g, 8, outer, t=BF16)
    dx, dw, db = ctx.grouped_mm_backward(dy, x, m, torch.tensor([0, rows], device="cuda"), gate=x)
    e, size = mm_exact(dy[ends], m.transpose(1, 2), torch.zeros(8, dtype=torch.int64, device="cuda"), None, False)
    open_ = x[ends] > 0
    close(dx[ends], e.masked_fill(~open_, 0.0), (2 * (outer + 2) * U * size).masked_fill(~open_, 0.0))
    close(dw[0], x[ends].double().t() @ dy[ends].double(), 2 * 8 * U * (x[ends].double().abs().t() @ dy[ends].double().abs()))
    close(db[0], dy[ends].double().sum(0), 2 * 8 * U * dy[ends].double().abs().sum(0))


def test_a_launch_of_more_workgroups_than_a_dimension_holds(ctx):   # noqa: F811
    """2^30 rows of few columns: 2^24 workgroups of 256 threads, one more than 2^32 threads in a line. (Neighbouring rows overlap in all but one element.)"""
    say("2^30 rows")
    rows, inner = 2 ** 30, 4
    g = generator(12)
    line = torch.randn(rows + inner - 1, generator=g, device="cuda", dtype=BF16)
    w = normal(g, 1, inner, 1, t=BF16)
    y = ctx.grouped_mm(line.as_strided((rows, inner), (1, 1)), w, torch.tensor([0, rows], device="cuda"))
    assert y.shape == (rows, 1)
    part = 2 ** 26
    for first in range(0, rows, part):
        terms = [line[first + j:first + j + part].float() * w[0, j, 0].float() for j in range(inner)]   # (exact: 8 bits by 8)
        size = sum(v.abs() for v in terms)
        # four terms in two orders, a rounding of the kernel's result
        assert ((y[first:first + part, 0].float() - sum(terms)).abs() <= (2 * (inner + 2) + inner) * U * size + 2.0 ** -8 * size).all(), first


def test_the_most_rows_by_group(ctx):   # noqa: F811
    """2^30 rows in 1,000 groups, the limits of the call but for 24 groups."""
    say("2^30 rows by group")
    rows, groups = 2 ** 30, 1000
    ids = torch.randint(-1, groups, (rows,), generator=generator(13), device="cuda", dtype=torch.int32)
    offsets, order = ctx.group_rows(ids, groups)
    of = torch.bincount(ids + 1, minlength=groups + 1)
    assert offsets.tolist() == [0] + torch.cumsum(of[1:], 0).tolist()
    part = 2 ** 26
    for first in range(0, rows, part):
        at = order[max(first - 1, 0):first + part].long()
        key = ids[at]
        key = torch.where(key < 0, groups, key)
        step = key[1:] - key[:-1]
        # by group, and ascending within a group: with the sizes of the groups, every row once
        assert (step >= 0).all() and (at[1:] > at[:-1])[step == 0].all() and at.min() >= 0 and at.max() < rows, first


def test_many_groups_captured_into_a_graph():
    """Groups whose counts need more LDS than a kernel has by itself, and the gradient of the weights in two launches."""
    say("graph of many groups")
    from paper_2506_22668_amd import Context
    stream = torch.cuda.Stream()
    mine, plain = Context("cuda:0", stream=stream), Context("cuda:0")
    rows, inner, outer, groups = 60_000, 128, 136, 1000

    def inputs(seed):
        g = generator(seed)
        return [torch.randint(-1, groups, (rows,), generator=g, device="cuda").int(), normal(g, rows, inner, t=BF16), normal(g, rows, outer, t=BF16),
                normal(g, groups, inner, outer, t=BF16, scale=0.1)]

    def run(c, ids, x, dy, w):
        offsets, order = c.group_rows(ids, groups)
        return [offsets, order, c.grouped_mm(x, w, offsets, order=order), *c.grouped_mm_backward(dy, x, w, offsets, order=order, gate=x)]

    held = inputs(1)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=stream):
        out = run(mine, *held)
    for seed in (2, 3, 4):
        for to, new in zip(held, inputs(seed)):
            to.copy_(new)
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(out, run(plain, *held))), seed
    mine.close()
    plain.close()


@pytest.mark.parametrize("t, element", [(F32, 0), (BF16, 1), (F16, 2)])
@pytest.mark.parametrize("rows, inner, outer, groups", [(90, 24, 40, 65), (2000, 24, 16, 600), (20_000, 64, 264, 65), (60_000, 64, 72, 1000)])
def test_offsets_that_do_not_ascend_stay_inside(ctx, t, element, rows, inner, outer, groups):   # noqa: F811
    """Every other group has all rows, and all have the same weights: a row of the product is right or left as it was, and nothing around the outputs changes."""
    say(f"offsets up and down {t} rows={rows} groups={groups}")
    lib, g = ctx.lib, generator(rows)
    x, dy = normal(g, rows, inner, t=t), normal(g, rows, outer, t=t)
    w = normal(g, 1, inner, outer, t=t, scale=inner ** -0.5).repeat(groups, 1, 1)
    offsets = torch.tensor([0 if k % 2 == 0 else rows for k in range(groups + 1)], device="cuda")
    want = ctx.grouped_mm(x, w[:1], torch.tensor([0, rows], device="cuda"))
    e, size = mm_exact(x, w[:1], torch.zeros(rows, dtype=torch.int64, device="cuda"), None, False)
    before, guard = 2 * (inner + 2) * U * size, 64

    def guarded(*shape, of=t):
        n = int(np.prod(shape))
        buf = torch.full((n + 2 * guard,), 3.0, dtype=of, device="cuda")
        return buf, buf[guard:guard + n].view(*shape)

    def untouched(buf):
        return (buf[:guard] == 3).all() and (buf[-guard:] == 3).all()

    outer_y, y = guarded(rows, outer)
    assert lib.ds_grouped_mm(ctx.h, element, rows, inner, outer, groups, x.data_ptr(), inner, w.data_ptr(), offsets.data_ptr(), None, None, 0,
                             y.data_ptr(), outer) == 0
    left = (y == 3).all(1) | (y == 0).all(1)   # (rows that some group's end leaves to no group are zeros)
    close(torch.where(left[:, None], want, y), e, before)
    assert untouched(outer_y)
    buffers = [guarded(rows, inner), guarded(groups, inner, outer), guarded(groups, outer, of=F32)]
    ws, ptr, n = ctx._workspace(lib.ds_grouped_mm_backward_workspace, element, rows, inner, outer, groups)
    assert lib.ds_grouped_mm_backward(ctx.h, element, rows, inner, outer, groups, dy.data_ptr(), outer, x.data_ptr(), inner, w.data_ptr(), offsets.data_ptr(),
                                      None, None, 0, buffers[0][1].data_ptr(), inner, buffers[1][1].data_ptr(), buffers[2][1].data_ptr(), ptr, n) == 0
    assert all(untouched(buf) for buf, _ in buffers)
    assert torch.equal(ctx.grouped_mm(x, w[:1], torch.tensor([0, rows], device="cuda")), want)
