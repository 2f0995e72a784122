"""The typed encoder's training state without a GPU: the operators written out in torch, its gradients against autograd, in the orders
of calls that a program makes."""
import pytest

from paper_2506_22668_amd.binding import DistShapError

torch = pytest.importorskip("torch")


class PlainContext:
    """What TypedEncoder calls of a Context, in 64 bits inside."""
    device = torch.device("cpu")

    def group_rows(self, ids, groups):
        key = torch.where((ids >= 0) & (ids < groups), ids, groups)
        return torch.searchsorted(key.sort(stable=True)[0].long(), torch.arange(groups + 1)), key.argsort(stable=True).int()

    def layer_norm(self, x, weight, bias, want_stats):
        v = x.double()
        mean = v.mean(1)
        rstd = 1 / torch.sqrt(v.var(1, unbiased=False) + 1e-5)
        return ((v - mean[:, None]) * rstd[:, None] * weight + bias).to(x.dtype), mean, rstd

    def layer_norm_backward(self, dy, x, mean, rstd, weight):
        hat, g = (x.double() - mean[:, None]) * rstd[:, None], dy.double() * weight
        dx = rstd[:, None] * (g - g.mean(1, keepdim=True) - hat * (g * hat).mean(1, keepdim=True))
        return dx.to(x.dtype), (dy * hat).sum(0).float(), dy.sum(0).float()

    def _groups(self, offsets, order):
        return [order[offsets[g]:offsets[g + 1]].long() for g in range(len(offsets) - 1)]

    def grouped_mm(self, x, w, offsets, order=None, bias=None, relu=False):
        y = torch.zeros(x.shape[0], w.shape[2], dtype=torch.float64)
        for g, at in enumerate(self._groups(offsets, order)):
            y[at] = x[at].double() @ w[g].double() + bias[g]
        return (y.clamp(min=0) if relu else y).to(x.dtype)

    def grouped_mm_backward(self, dy, x, w, offsets, order=None, gate=None):
        dx, dw, db = torch.zeros(x.shape, dtype=torch.float64), torch.zeros(w.shape, dtype=torch.float64), torch.zeros(w.shape[0], w.shape[2])
        for g, at in enumerate(self._groups(offsets, order)):
            dx[at] = dy[at].double() @ w[g].double().t()
            dw[g], db[g] = x[at].double().t() @ dy[at].double(), dy[at].double().sum(0)
        if gate is not None:
            dx[~(gate > 0)] = 0
        return dx.to(x.dtype), dw.to(x.dtype), db

    def dropout(self, x, p, seed, tag=0, residual=None):
        g = torch.Generator()
        g.manual_seed((seed * 31 + tag) % 2 ** 31)
        y = torch.where(torch.rand(x.shape, generator=g) >= p, x / (1 - p) if p < 1 else x, torch.zeros_like(x))
        return y if residual is None else y + residual


WIDTH, TYPES = 12, 2


def encoder(dtype=torch.float32):
    from paper_2506_22668_amd.encoder import TypedEncoder
    return TypedEncoder(PlainContext(), TYPES, WIDTH, 20, depth=2, dtype=dtype, p=0.25, seed=3)


def batch(seed, rows):
    g = torch.Generator()
    g.manual_seed(seed)
    return torch.randn(rows, WIDTH, generator=g), torch.randint(-1, TYPES, (rows,), generator=g).int(), torch.randn(rows, WIDTH, generator=g)


def wanted(enc, x, kind, dy, step):
    """dx and the gradients of the parameters by autograd."""
    x = x.double().requires_grad_(True)
    first, params = x, []
    for tag, b in enumerate(enc.blocks):
        q = {k: v.double().requires_grad_(True) for k, v in b.items()}
        params.append(q)
        y = torch.nn.functional.layer_norm(x, (WIDTH,), q["gain"], q["shift"])
        out = torch.zeros_like(x)
        for k in range(TYPES):
            at = (kind == k).nonzero()[:, 0]
            out = out.index_put((at,), (y[at] @ q["w1"][k] + q["b1"][k]).clamp(min=0) @ q["w2"][k] + q["b2"][k])
        x = x + enc.ctx.dropout(torch.ones_like(x), 0.25, 3 + (step << 32), tag) * out
    x.backward(dy.double())
    return first.grad, [{k: v.grad for k, v in q.items()} for q in params]


def agrees(dx, grads, want):
    assert len(grads) == len(want[1])
    assert torch.allclose(dx.double(), want[0], rtol=1e-4, atol=1e-5)
    for got, q in zip(grads, want[1]):
        for k, v in q.items():
            assert torch.allclose(got[k].double(), v, rtol=1e-4, atol=1e-4), k


def test_gradients_of_a_training_step():
    enc, (x, kind, dy) = encoder(), batch(1, 30)
    want = wanted(enc, x, kind, dy, 5)
    enc.forward(x, kind, train=True, step=5)
    agrees(enc.backward(dy), enc.grads, want)
    before = [{k: v.clone() for k, v in b.items()} for b in enc.blocks]
    enc.update(0.5)
    for b, old, g in zip(enc.blocks, before, enc.grads):
        for k in b:
            assert torch.allclose(b[k], old[k] - 0.5 * g[k])


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_an_evaluation_leaves_the_training_state_alone(dtype):
    enc, (x, kind, dy), (other, other_kind, _) = encoder(dtype), batch(1, 30), batch(2, 17)
    enc.forward(x, kind, train=True, step=5)
    want, want_grads = enc.backward(dy), enc.grads
    enc.forward(x, kind, train=True, step=5)
    enc.forward(other, other_kind)
    got = enc.backward(dy)
    assert torch.equal(got, want) and len(enc.grads) == len(want_grads) == 2
    for a, b in zip(enc.grads, want_grads):
        assert all(torch.equal(a[k], b[k]) for k in b)


def test_a_backward_pass_needs_a_training_forward_of_its_own():
    enc, (x, kind, dy) = encoder(), batch(1, 30)
    with pytest.raises(DistShapError):
        enc.backward(dy)
    enc.forward(x, kind)
    with pytest.raises(DistShapError):
        enc.backward(dy)
    with pytest.raises(DistShapError):
        enc.update(0.1)
    enc.forward(x, kind, train=True)
    with pytest.raises(DistShapError):
        enc.update(0.1)               # (no gradients yet)
    enc.backward(dy)
    with pytest.raises(DistShapError):
        enc.backward(dy)              # (its forward has had its own)


def test_two_training_forwards_are_told_apart():
    enc, (x, kind, dy), (other, other_kind, other_dy) = encoder(), batch(1, 30), batch(2, 30)
    want, other_want = wanted(enc, x, kind, dy, 0), wanted(enc, other, other_kind, other_dy, 1)
    enc.forward(x, kind, train=True)
    first = enc.state
    enc.forward(other, other_kind, train=True, step=1)
    second = enc.state
    with pytest.raises(DistShapError):
        enc.backward(dy)              # (of which?)
    agrees(enc.backward(dy, first), enc.grads, want)
    agrees(enc.backward(other_dy, second), enc.grads, other_want)
    enc.forward(x, kind, train=True)
    agrees(enc.backward(dy), enc.grads, want)


@pytest.mark.parametrize("change", ["input", "update", "weight"])
def test_what_a_backward_pass_reads_must_not_have_changed(change):
    """fp32 weights and inputs are read where they lie: overwritten, they would give the gradient of another function."""
    enc, (x, kind, dy) = encoder(), batch(1, 30)
    enc.forward(x, kind, train=True)
    enc.backward(dy)
    enc.forward(x, kind, train=True)
    if change == "input":
        x.mul_(2)
    elif change == "update":
        enc.update(0.1)
    else:
        enc.blocks[1]["w2"].zero_()
    with pytest.raises(DistShapError):
        enc.backward(dy)


def test_a_gradient_of_other_rows_is_refused():
    enc, (x, kind, dy) = encoder(), batch(1, 30)
    enc.forward(x, kind, train=True)
    with pytest.raises(DistShapError):
        enc.backward(dy[:29])
