"""The routed encoder without a GPU: its operators written out in torch, its gradients against autograd, in the orders of calls that a program makes."""
import pytest

from paper_2506_22668_amd.binding import DistShapError
from tests.test_encoder import PlainContext

torch = pytest.importorskip("torch")


class Plain(PlainContext):
    """What RoutedEncoder calls of a Context, in 64 bits inside."""

    def _order(self, x, order):
        return torch.arange(x.shape[0]) if order is None else order

    def grouped_mm(self, x, w, offsets, order=None, bias=None, relu=False):
        return super().grouped_mm(x, w, offsets, self._order(x, order), torch.zeros(w.shape[0], w.shape[2]) if bias is None else bias, relu)

    def grouped_mm_backward(self, dy, x, w, offsets, order=None, gate=None):
        return super().grouped_mm_backward(dy, x, w, offsets, self._order(x, order), gate)

    def embed(self, table, ids, scale=1.0, dtype=None):
        there = (ids >= 0) & (ids < table.shape[0])
        return torch.where(there[:, None], table[ids.clamp(0, table.shape[0] - 1).long()].double() * scale, 0.0).to(dtype)

    def embed_backward(self, dy, ids, vocab, scale=1.0, dtype=None):
        there = (ids >= 0) & (ids < vocab)
        return torch.zeros(vocab, dy.shape[1], dtype=torch.float64).index_add_(0, ids[there].long(), dy[there].double() * scale).to(dtype)

    def route(self, x, k, renorm):
        p = torch.softmax(x.double(), 1)
        ids = torch.sort(x, dim=1, descending=True, stable=True)[1][:, :k]
        w = p.gather(1, ids)
        w = w / w.sum(1, keepdim=True) if renorm else w
        counts = torch.cat([torch.bincount(ids.reshape(-1), minlength=x.shape[1]), torch.tensor([x.shape[0]])])
        loss = x.shape[1] * (counts[:-1] / counts[:-1].sum() * p.mean(0)).sum()
        return ids.t().int(), w.t().float(), counts, loss.float(), torch.logsumexp(x.double(), 1)

    def route_backward(self, x, lse, ids, counts, dweights=None, dloss=None, renorm=False):
        with torch.enable_grad():
            z = x.double().detach().requires_grad_(True)
            p = torch.softmax(z, 1)
            w = p.gather(1, ids.t().long())
            w = w / w.sum(1, keepdim=True) if renorm else w
            loss = x.shape[1] * (counts[:-1] / counts[:-1].sum() * p.mean(0)).sum()
            ((w.t() * dweights).sum() + loss * dloss).backward()
        return z.grad.to(x.dtype)


NODES, EXPERTS, WIDTH, K = 9, 3, 10, 2


def encoder(dtype=torch.float32):
    from paper_2506_22668_amd.encoder import RoutedEncoder
    return RoutedEncoder(Plain(), NODES, EXPERTS, WIDTH, 14, depth=2, k=K, dtype=dtype, p=0.25, seed=3)


def batch(seed, rows=20):
    g = torch.Generator()
    g.manual_seed(seed)
    return torch.randint(-1, NODES + 1, (rows,), generator=g).int(), torch.randn(rows, WIDTH, generator=g)


def wanted(enc, ids, dy, step, balance):
    """The gradients of the parameters by autograd, the choices those of the scores."""
    table = enc.table.double().requires_grad_(True)
    there = (ids >= 0) & (ids < NODES)
    x = torch.where(there[:, None], table[ids.clamp(0, NODES - 1).long()] * enc.scale, 0.0)
    params, loss = [], 0.0
    for tag, b in enumerate(enc.blocks):
        q = {k: v.double().requires_grad_(True) for k, v in b.items()}
        params.append(q)
        y = torch.nn.functional.layer_norm(x, (WIDTH,), q["gain"], q["shift"])
        scores = y @ q["router"]
        p = torch.softmax(scores, 1)
        chosen = torch.sort(scores, dim=1, descending=True, stable=True)[1][:, :K]   # (of equal scores the first: a row of no id has nothing else)
        w = p.gather(1, chosen)
        w = w / w.sum(1, keepdim=True)
        counts = torch.bincount(chosen.reshape(-1), minlength=EXPERTS)
        loss = loss + EXPERTS * (counts / counts.sum() * p.mean(0)).sum()
        total = torch.zeros_like(x)
        for j in range(K):
            h = torch.relu(torch.einsum("rc,rcd->rd", y, q["w1"][chosen[:, j]]) + q["b1"][chosen[:, j]])   # (closed at zero, as the gate is)
            total = total + w[:, j:j + 1] * (torch.einsum("rc,rcd->rd", h, q["w2"][chosen[:, j]]) + q["b2"][chosen[:, j]])
        x = x + enc.ctx.dropout(torch.ones_like(x), 0.25, 3 + (step << 32), tag) * total
    ((x * dy.double()).sum() + balance * loss).backward()
    return x, loss, table.grad, [{k: v.grad for k, v in q.items()} for q in params]


def near(a, b, what):
    # (fp32 roundings of a chain of two blocks: sixteen a block and way, of the largest entry)
    assert (a.double() - b).abs().max() <= 64 * 2.0 ** -24 * max(1.0, b.abs().max().item()) * WIDTH, what


@pytest.mark.parametrize("balance", [0.0, 0.7])
def test_gradients_are_those_of_autograd(balance):
    enc = encoder()
    ids, dy = batch(1)
    out = enc.forward(ids, train=True, step=2)
    enc.backward(dy, balance=balance)
    x, loss, dtable, grads = wanted(enc, ids, dy, 2, balance)
    near(out, x.detach(), "out")
    near(enc.balance, loss.detach(), "balance")
    near(enc.dtable, dtable, "table")
    for got, want in zip(enc.grads, grads):
        assert set(got) == set(want)
        for k in want:
            near(got[k], want[k], k)
    assert [int(c[-1]) for c in enc.counts] == [20, 20]


def test_a_step_changes_the_parameters_along_their_gradients():
    enc = encoder()
    ids, dy = batch(2)
    before = enc.table.clone(), [{k: v.clone() for k, v in b.items()} for b in enc.blocks]
    enc.forward(ids, train=True)
    enc.backward(dy)
    enc.update(0.5)
    assert torch.equal(enc.table, before[0] - 0.5 * enc.dtable)
    for b, was, g in zip(enc.blocks, before[1], enc.grads):
        for k in b:
            assert torch.equal(b[k], was[k] - 0.5 * g[k].float())


def test_orders_of_calls_that_do_not_fit_are_refused():
    enc = encoder()
    ids, dy = batch(3)
    with pytest.raises(DistShapError):
        enc.update(0.1)
    with pytest.raises(DistShapError):
        enc.backward(dy)
    enc.forward(ids, train=True)
    first = enc.state
    enc.forward(ids)                      # an evaluation leaves the training state alone
    assert enc.state is first
    with pytest.raises(DistShapError):
        enc.backward(dy[:-1])
    enc.forward(ids, train=True)
    with pytest.raises(DistShapError):
        enc.backward(dy)                  # of which forward?
    with pytest.raises(DistShapError):
        enc.update(0.1)                   # a backward pass that failed leaves no gradients
    enc.backward(dy, state=first)
    enc.update(0.1)
    enc.forward(ids, train=True)
    ids[0] = 1 - ids[0]                   # the ids of the step have been changed
    with pytest.raises(DistShapError):
        enc.backward(dy)
