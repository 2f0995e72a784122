"""The typed encoder (operators on rows run together) against the same blocks written out in 64 bits, and a short training."""
import pytest

from tests.gpu_common import say

pytestmark = pytest.mark.gpu
torch = pytest.importorskip("torch")


def _plain(enc, x, kind, masks, gates):
    """The blocks in 64 bits, differentiable; masks: what each block's dropout multiplies by; gates: where its ReLU was open. (A value
    that rounding takes across zero opens or closes it: the gradient is that of the function as it was evaluated.)"""
    params = []
    x = x.double().requires_grad_(True)
    first = x
    for b, mask, gate in zip(enc.blocks, masks, gates):
        q = {k: v.double().requires_grad_(True) for k, v in b.items()}
        params.append(q)
        mean = x.mean(1, keepdim=True)
        y = (x - mean) / torch.sqrt((x - mean).square().mean(1, keepdim=True) + 1e-5) * q["gain"] + q["shift"]
        out = torch.zeros_like(x)
        for k in range(enc.types):
            at = kind == k
            out = out.index_put((at.nonzero()[:, 0],), ((y[at] @ q["w1"][k] + q["b1"][k]) * gate[at]) @ q["w2"][k] + q["b2"][k])
        x = x + mask * out
    return first, x, params


# A chain of two blocks: five roundings a block forward and back (norm, two products, dropout's sum; the same again), each half a
# step of the type relative to the size of what it rounds; the largest entry of a whole tensor is held to sixteen of them, its mean to four.
@pytest.mark.parametrize("t, steps", [(torch.float32, 512), (torch.bfloat16, 16), (torch.float16, 16)])
def test_gradients_of_the_encoder(t, steps):
    from paper_2506_22668_amd import Context
    from paper_2506_22668_amd.encoder import TypedEncoder
    say(f"encoder gradients {t}")
    ctx = Context("cuda:0")
    g = torch.Generator(device="cuda")
    g.manual_seed(2)
    n, width = 333, 40
    x, c = torch.randn(n, width, generator=g, device="cuda"), torch.randn(n, width, generator=g, device="cuda").to(t).float()
    x = x.to(t).float()
    kind = torch.randint(-1, 3, (n,), generator=g, device="cuda").int()
    enc = TypedEncoder(ctx, 3, width, 56, depth=2, dtype=t, p=0.25, seed=9)
    for b in enc.blocks:   # (what the products see)
        for k in ("w1", "w2"):
            b[k] = b[k].to(t).float()
    out = enc.forward(x, kind, train=True, step=4)
    dx = enc.backward(c)
    ones = torch.ones(n, width, device="cuda")
    masks = [ctx.dropout(ones, 0.25, 9 + (4 << 32), tag).double() for tag in range(2)]
    first, want, params = _plain(enc, x, kind, masks, [(kept[2] > 0).double() for kept in enc._kept])
    want.backward(c.double())
    bound = steps * torch.finfo(t).eps / 2

    def near(a, b):
        off, size = (a.double() - b).abs(), b.abs().max().item()
        assert torch.isfinite(a).all() and off.max().item() <= bound * size and off.mean().item() <= bound / 4 * size
    near(out, want.detach())
    near(dx, first.grad)
    for got, q in zip(enc.grads, params):
        for k, v in q.items():
            near(got[k], v.grad)
    assert torch.equal(enc.forward(x, kind)[kind < 0], x.to(t)[kind < 0])   # rows of no type pass through
    ctx.close()


def test_the_example_learns_and_explains(capsys):
    from paper_2506_22668_amd import encoder
    say("encoder example")
    encoder.main(nodes=600, steps=40)
    lines = capsys.readouterr().out.splitlines()
    errors = [float(line.rsplit(" ", 1)[1]) for line in lines if line.startswith("step")]
    assert errors[-1] < 0.7 * errors[0], errors
    assert "node 5 is of class" in lines[-1]
