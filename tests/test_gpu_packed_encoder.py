"""RoutedEncoder with its training rows in 8 bits, on the GPU: its gradients against the backward pass written out in 64 bits on the rows that were kept.

Tolerances are those of tests/test_gpu_learning.py for the encoder that keeps its rows as they are: a chain of two blocks, eight roundings of the type a block and way, each half a step
relative to the size of what it rounds, the largest entry of a tensor held to 32 of them and its mean to eight. The codes themselves are read without a rounding of the type
(4 bits of a value, a power of two), so they add nothing."""
import pytest

from tests.encoder_steps import routed_backward
from tests.gpu_common import say
from tests.test_gpu_features import BF16, F16, F32, generator, normal

pytestmark = pytest.mark.gpu
torch = pytest.importorskip("torch")


@pytest.fixture(scope="module")
def ctx():
    from paper_2506_22668_amd import Context
    c = Context("cuda:0")
    yield c
    c.close()


@pytest.mark.parametrize("t, steps", [(F32, 1024), (BF16, 32), (F16, 32)])
@pytest.mark.parametrize("rows, width, hidden", [(333, 40, 56), (2500, 64, 96)])
@pytest.mark.parametrize("balance", [0.0, 2.0])
def test_gradients_of_the_routed_encoder_that_keeps_8_bits(ctx, t, steps, rows, width, hidden, balance):
    from paper_2506_22668_amd import Packed
    from paper_2506_22668_amd.encoder import RoutedEncoder
    say(f"packed routed encoder gradients {t} rows={rows} balance={balance}")
    g = generator(2)
    enc = RoutedEncoder(ctx, 70, 5, width, hidden, depth=2, k=2, dtype=t, p=0.25, seed=9, packed=True)
    ids = torch.randint(-1, 71, (rows,), generator=g, device="cuda").int()
    c = normal(g, rows, width).to(t)
    enc.forward(ids, train=True, step=4)
    state = enc.state
    enc.backward(c, balance=balance)
    ones = torch.ones(rows, width, device="cuda")
    masks = [ctx.dropout(ones, 0.25, 9 + (4 << 32), tag) for tag in range(2)]
    assert all(isinstance(m, Packed) for block in state.blocks for m in [block[1]] + [m for part in block[13] for m in part[:2]])
    dtable, grads = routed_backward(enc, state, c, balance, masks, lambda m: ctx.unpack_rows(m).double())
    bound = steps * torch.finfo(t).eps / 2

    def near(a, b, what):
        off, size = (a.double() - b).abs(), b.abs().max().item()
        assert torch.isfinite(a).all() and off.max().item() <= bound * size and off.mean().item() <= bound / 4 * size, (what, off.max().item() / size / bound)
    near(enc.dtable, dtable, "table")
    for got, want in zip(enc.grads, grads):
        assert set(got) == set(want)
        for name, v in want.items():
            near(got[name], v, name)
