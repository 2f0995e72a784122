"""Embeddings, the router and rows in 8 bits together, as the encoders use them: gradients against the same blocks written out in 64 bits, the calls on other
streams and captured into graphs, and the example."""
import pytest

from tests.gpu_common import say
from tests.test_gpu_features import BF16, F16, F32, U, close, generator, normal

pytestmark = pytest.mark.gpu
torch = pytest.importorskip("torch")


@pytest.fixture(scope="module")
def ctx():
    from paper_2506_22668_amd import Context
    c = Context("cuda:0")
    yield c
    c.close()


def _plain(enc, ids, choices, masks, gates):
    """The blocks in 64 bits, differentiable; choices, masks and gates: which experts were chosen, what dropout multiplies by, where each ReLU was open."""
    table = enc.table.double().requires_grad_(True)
    there = (ids >= 0) & (ids < table.shape[0])
    x = torch.where(there[:, None], table[ids.clamp(0, table.shape[0] - 1).long()] * enc.scale, 0.0)
    params, loss = [], 0.0
    for b, chosen, mask, gate in zip(enc.blocks, choices, masks, gates):
        q = {k: v.double().requires_grad_(True) for k, v in b.items()}
        params.append(q)
        mean = x.mean(1, keepdim=True)
        y = (x - mean) / torch.sqrt((x - mean).square().mean(1, keepdim=True) + 1e-5) * q["gain"] + q["shift"]
        p = torch.softmax(y @ q["router"], 1)
        w = p.gather(1, chosen.t().long())
        w = w / w.sum(1, keepdim=True)
        share = torch.bincount(chosen.reshape(-1).long(), minlength=enc.types).double() / chosen.numel()
        loss = loss + enc.types * (share * p.mean(0)).sum()
        total = torch.zeros_like(x)
        for j in range(enc.k):
            e = chosen[j].long()
            part = torch.zeros_like(x)
            for k in range(enc.types):
                at = (e == k).nonzero()[:, 0]
                part = part.index_put((at,), ((y[at] @ q["w1"][k] + q["b1"][k]) * gate[j][at]) @ q["w2"][k] + q["b2"][k])
            total = total + w[:, j:j + 1] * part
        x = x + mask * total
    return x, loss, table, params


# A chain of two blocks: eight roundings a block forward and back (lookup, norm, scores, two products for each choice, their sum, dropout's; the same again), each half
# a step of the type relative to the size of what it rounds; the largest entry of a whole tensor is held to 32 of them, its mean to eight. What the scores' roundings do to
# the weights goes through the softmax's slope, at most 1, and is among them.
@pytest.mark.parametrize("t, steps", [(F32, 1024), (BF16, 32), (F16, 32)])
def test_gradients_of_the_routed_encoder(ctx, t, steps):
    from paper_2506_22668_amd.encoder import RoutedEncoder
    say(f"routed encoder gradients {t}")
    g = generator(2)
    n, width, experts = 333, 40, 5
    enc = RoutedEncoder(ctx, 70, experts, width, 56, depth=2, k=2, dtype=t, p=0.25, seed=9)
    for b in enc.blocks:   # (what the products see)
        for k in ("w1", "w2", "router"):
            b[k] = b[k].to(t).float()
    ids = torch.randint(-1, 71, (n,), generator=g, device="cuda").int()
    c = normal(g, n, width).to(t).float()
    out = enc.forward(ids, train=True, step=4)
    state = enc.state
    enc.backward(c, balance=2.0)
    ones = torch.ones(n, width, device="cuda")
    masks = [ctx.dropout(ones, 0.25, 9 + (4 << 32), tag).double() for tag in range(2)]
    choices = [kept[9] for kept in state.blocks]
    gates = [[(part[0] > 0).double() for part in kept[13]] for kept in state.blocks]
    want, loss, table, params = _plain(enc, ids, choices, masks, gates)
    ((want * c.double()).sum() + 2.0 * loss).backward()
    bound = steps * torch.finfo(t).eps / 2

    def near(a, b, what):
        off, size = (a.double() - b).abs(), b.abs().max().item()
        assert torch.isfinite(a).all() and off.max().item() <= bound * size and off.mean().item() <= bound / 4 * size, (what, off.max().item() / size / bound)
    near(out, want.detach(), "out")
    near(enc.balance, loss.detach(), "balance")
    near(enc.dtable, table.grad, "table")
    for got, q in zip(enc.grads, params):
        assert set(got) == set(q)
        for k, v in q.items():
            near(got[k], v.grad, k)


@pytest.mark.parametrize("t", [F32, BF16, F16])
def test_encoders_that_keep_8_bits(ctx, t):
    """What goes out is what goes out without; the weights' gradients are those of the rows that the codes stand for."""
    from paper_2506_22668_amd import Packed
    from paper_2506_22668_amd.encoder import RoutedEncoder, TypedEncoder
    say(f"packed encoders {t}")
    g = generator(3)
    x, kind, c = normal(g, 200, 48), torch.randint(-1, 3, (200,), generator=g, device="cuda").int(), normal(g, 200, 48).to(t)
    one, other = (TypedEncoder(ctx, 3, 48, 72, depth=1, dtype=t, p=0.2, seed=5, packed=packed) for packed in (False, True))
    assert torch.equal(one.forward(x, kind, train=True), other.forward(x, kind, train=True))
    one.backward(c)
    other.backward(c)
    _, y, h, _, _, w1, w2, offsets, order, _, tag = other._kept[0]
    assert isinstance(y, Packed) and isinstance(h, Packed)
    y, h = ctx.unpack_rows(y, t), ctx.unpack_rows(h, t)
    dout = ctx.dropout(c, 0.2, other.state.seed, tag)
    dh = ctx.grouped_mm_backward(dout, h, w2, offsets, order=order, gate=h)[0]
    got, plain = other.grads[0], one.grads[0]
    assert torch.equal(got["b2"], plain["b2"]) and torch.equal(got["b1"], plain["b1"])   # (the gate of the codes is the gate)
    for k in range(3):
        at = kind == k
        for name, rows, dy in (("w2", h, dout), ("w1", y, dh)):
            rows, dy, n = rows[at].double(), dy[at].double(), int(at.sum())
            close(got[name][k], rows.t() @ dy, 2 * n * U * (rows.abs().t() @ dy.abs()))
    ids = torch.randint(0, 30, (200,), generator=g, device="cuda").int()
    a, b = (RoutedEncoder(ctx, 30, 4, 48, 72, depth=2, dtype=t, p=0.2, seed=6, packed=packed) for packed in (False, True))
    assert torch.equal(a.forward(ids, train=True), b.forward(ids, train=True)) and torch.equal(a.balance, b.balance)
    b.backward(c, balance=1.0)
    b.update(0.01)
    assert torch.isfinite(b.dtable).all() and all(torch.isfinite(v).all() for grads in b.grads for v in grads.values())


# ---- the calls as a program makes them --------------------------------------------------------------------------------------------

def _all(ctx, s, experts=6):
    x = ctx.embed(s["table"], s["ids"], scale=4.0, dtype=BF16)
    scores = ctx.grouped_mm(x, s["router"], s["whole"])
    ids, weights, counts, loss, lse = ctx.route(scores, 2, renorm=True)
    offsets, order = ctx.group_rows(ids[0], experts)
    kept = ctx.pack_rows(x)
    h = ctx.grouped_mm(x, s["w"], offsets, order=order, relu=True)
    held = ctx.pack_rows(h)
    dx, dw, db = ctx.grouped_mm_backward(s["dy"], kept, s["w"], offsets, order=order, gate=kept)
    dh = ctx.grouped_mm_backward(s["dy"], held, s["w"], offsets, order=order, gate=held)[0]
    dscores = ctx.route_backward(scores, lse, ids, counts, dweights=s["dweights"], dloss=s["dloss"], renorm=True)
    dtable = ctx.embed_backward(dx, s["ids"], s["table"].shape[0], scale=4.0, dtype=F32)
    return [x, scores, ids, weights, counts, loss, lse, offsets, order, kept.codes.view(torch.uint8), kept.scales, ctx.unpack_rows(held, BF16), dx, dw, db, dh, dscores, dtable]


def _inputs(rows, vocab, seed):
    g = generator(seed)
    return dict(table=normal(g, vocab, 136), ids=torch.randint(-1, vocab, (rows,), generator=g, device="cuda").int(), router=normal(g, 1, 136, 6, t=BF16, scale=0.1),
                w=normal(g, 6, 136, 136, t=BF16, scale=0.1), dy=normal(g, rows, 136, t=BF16), dweights=normal(g, 2, rows), dloss=normal(g, 1),
                whole=torch.tensor([0, rows], device="cuda"))


SIZES = [(50, 70), (9_000, 300), (70_000, 200_000), (20_000, 600_000)]


@pytest.mark.parametrize("rows, vocab", SIZES)
def test_calls_on_another_stream_than_the_contexts(ctx, rows, vocab):
    say(f"learning streams rows={rows}")
    from paper_2506_22668_amd import Context
    s = _inputs(rows, vocab, 1)
    want = _all(ctx, s)
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    other = Context("cuda:0", stream=torch.cuda.Stream())
    for c in (ctx, other):
        with torch.cuda.stream(side):
            fresh = {k: torch.zeros_like(v) for k, v in s.items()}
            for k in s:                       # (inputs made on the side stream right before the calls)
                fresh[k].copy_(s[k])
            got = [v.clone() for v in _all(c, fresh)]    # (and outputs used there right behind them)
        side.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(got, want))
    other.close()


@pytest.mark.parametrize("rows, vocab", SIZES)
def test_calls_captured_into_a_graph(ctx, rows, vocab):
    say(f"learning graph rows={rows}")
    from paper_2506_22668_amd import Context
    stream = torch.cuda.Stream()
    mine = Context("cuda:0", stream=stream)
    s = _inputs(rows, vocab, 2)
    torch.cuda.synchronize()
    with torch.cuda.stream(stream):
        _all(mine, s)
    stream.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=stream):
        out = _all(mine, s)
    for seed in (3, 4, 5, 6):
        new = _inputs(rows, vocab, seed)
        for k in s:
            s[k].copy_(new[k])
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        want = _all(ctx, s)                  # (eager work between the replays)
        assert all(torch.equal(a, b) for a, b in zip(out, want)), seed
    mine.close()


@pytest.mark.parametrize("rows, vocab", [(9_000, 300), (70_000, 200_000)])
def test_two_graphs_replayed_in_turn(ctx, rows, vocab):
    """Two captures with workspaces of their own."""
    say(f"learning two graphs rows={rows}")
    from paper_2506_22668_amd import Context
    stream = torch.cuda.Stream()
    mine = Context("cuda:0", stream=stream)
    inputs, graphs, outs = [_inputs(rows, vocab, 7), _inputs(rows // 2, vocab, 8)], [], []
    torch.cuda.synchronize()
    for s in inputs:
        with torch.cuda.stream(stream):
            _all(mine, s)
        stream.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=stream):
            outs.append(_all(mine, s))
        graphs.append(graph)
    want = [_all(ctx, s) for s in inputs]
    torch.cuda.synchronize()
    for which in (0, 1, 0, 1, 1, 0):
        graphs[which].replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(outs[which], want[which])), which
    mine.close()


def test_gradients_are_calls_of_their_own(ctx):
    """Where autograd follows an input, its backward pass fails and leaves no gradient out."""
    say("learning autograd")
    from paper_2506_22668_amd import DistShapError
    g = generator(9)
    table, scores = normal(g, 5, 8).requires_grad_(True), normal(g, 6, 4).requires_grad_(True)
    ids = torch.tensor([0, 3, 4], device="cuda").int()
    x, w, offsets = normal(g, 6, 4).requires_grad_(True), normal(g, 1, 4, 4), torch.tensor([0, 6], device="cuda")
    kept = ctx.pack_rows(x)
    for value in (ctx.embed(table, ids).sum(), ctx.route(scores, 2)[1].sum(), ctx.route(scores, 2)[3], ctx.unpack_rows(kept).sum(),
                  ctx.grouped_mm_backward(normal(g, 6, 4), kept, w, offsets, gate=kept)[1].sum()):
        with pytest.raises(DistShapError):
            value.backward()
    with torch.no_grad():
        assert not ctx.embed(table, ids).requires_grad


@pytest.mark.parametrize("packed", [False, True])
@pytest.mark.parametrize("rows", [0, 1])
def test_steps_of_no_row_and_of_one(ctx, rows, packed):
    from paper_2506_22668_amd.encoder import RoutedEncoder
    say(f"routed encoder rows={rows} packed={packed}")
    enc = RoutedEncoder(ctx, 5, 3, 16, 24, depth=2, k=2, dtype=F32, p=0.0, packed=packed)
    ids = torch.full((rows,), 3, device="cuda").int()
    out = enc.forward(ids, train=True)
    assert out.shape == (rows, 16) and [int(c[-1]) for c in enc.counts] == [rows, rows]
    enc.backward(torch.ones_like(out), balance=1.0)
    came = enc.dtable.any(1).tolist()
    assert came == [False, False, False, rows == 1, False] and torch.isfinite(enc.dtable).all()
    for grads in enc.grads:
        for k, v in grads.items():
            assert torch.isfinite(v).all() and (rows == 1 or not v.any()), k
    enc.update(0.1)


@pytest.mark.parametrize("t", [F32, BF16, F16])
def test_gates_that_are_one_row_for_all_and_end_inside_a_piece(ctx, t):
    """Gates of rows and of codes, the last rows' pieces reaching over the end of the matrix."""
    say(f"gates {t}")
    g = generator(11)
    rows, inner, outer = 3001, 259, 64
    x, dy, w = normal(g, rows, inner, t=t).relu(), normal(g, rows, outer, t=t), normal(g, 2, inner, outer, t=t, scale=0.1)
    order = torch.randperm(rows, generator=g, device="cuda").int()
    offsets = torch.tensor([0, 1000, rows], device="cuda")
    open_ = ctx.grouped_mm_backward(dy, x, w, offsets, order=order)[0]
    for gate in (x, x[:1].expand(rows, inner), x[-1:].expand(rows, inner)):
        want = torch.where(gate > 0, open_, torch.zeros_like(open_))
        assert torch.equal(ctx.grouped_mm_backward(dy, x, w, offsets, order=order, gate=gate)[0], want)
        kept = ctx.pack_rows(x)
        held = ctx.pack_rows(gate.contiguous()) if gate is x else ctx.pack_rows(gate[:1].contiguous())
        if gate is not x:
            held = type(held)(held.codes.view(torch.uint8).expand(rows, inner).view(torch.float8_e4m3fn), held.scales.expand(rows, held.scales.shape[1]))
        assert torch.equal(ctx.grouped_mm_backward(dy, kept, w, offsets, order=order, gate=held)[0], want)


def test_the_example_runs(capsys):
    from paper_2506_22668_amd import encoder
    say("ids example")
    encoder.main_ids(nodes=300, width=24, steps=12)
    lines = capsys.readouterr().out.splitlines()
    assert sum(line.startswith("step") for line in lines) == 3 and "node 5 is of class" in lines[-1]
    assert sum(int(v) for v in lines[-2].split("[")[1].rstrip("]").split(",")) == 2 * 600   # (two experts for each of the step's rows)
