"""Encoders that keep their training rows in 8 bits, without a GPU: the gradients are those of the formulas on the rows that were kept."""
import pytest

from paper_2506_22668_amd import Packed
from tests.encoder_steps import routed_backward
from tests.test_routed_encoder import EXPERTS, K, NODES, WIDTH, Plain, batch, near

torch = pytest.importorskip("torch")


class PlainPacked(Plain):
    """With rows in 8 bits: the nearest e4m3 number of a block's 32 values over the smallest power of two that leaves them at or below 448, none but 0 becoming 0."""

    def pack_rows(self, x):
        rows, cols = x.shape
        v = torch.zeros(rows, (cols + 31) // 32 * 32, dtype=torch.float64)
        v[:, :cols] = x
        v = v.view(rows, -1, 32)
        top = v.abs().amax(2)
        scales = torch.where(top > 0, torch.ceil(torch.log2(top.clamp(min=1e-30) / 448)) + 127, 127.0)
        q = v / torch.exp2(scales - 127)[:, :, None]
        q = torch.where((q != 0) & (q.abs() < 2.0 ** -9), q.sign() * 2.0 ** -9, q)
        return Packed(q.view(rows, -1)[:, :cols].float().to(torch.float8_e4m3fn), scales.to(torch.uint8))

    def unpack_rows(self, packed, dtype=torch.float32):
        power = torch.exp2(packed.scales.double() - 127).repeat_interleave(32, 1)[:, :packed.codes.shape[1]]
        return (packed.codes.double() * power).to(dtype)

    def grouped_mm_backward(self, dy, x, w, offsets, order=None, gate=None):
        there = lambda a: self.unpack_rows(a, torch.float64) if isinstance(a, Packed) else a   # noqa: E731
        dx, dw, db = super().grouped_mm_backward(dy, there(x), w, offsets, order, there(gate))
        return dx.to(dy.dtype), dw.to(w.dtype), db


def encoder(depth=2):
    from paper_2506_22668_amd.encoder import RoutedEncoder
    return RoutedEncoder(PlainPacked(), NODES, EXPERTS, WIDTH, 40, depth=depth, k=K, dtype=torch.float32, p=0.25, seed=3, packed=True)


@pytest.mark.parametrize("balance", [0.0, 0.7])
def test_gradients_are_those_of_the_rows_that_were_kept(balance):
    enc = encoder()
    ids, dy = batch(4)
    enc.forward(ids, train=True, step=2)
    state = enc.state
    kept = [state.blocks[0][1]] + [m for part in state.blocks[0][13] for m in part[:2]]   # normalised rows, and of each choice the hidden ones and what came out
    assert all(isinstance(m, Packed) for m in kept)
    enc.backward(dy, balance=balance)
    values = lambda m: enc.ctx.unpack_rows(m, torch.float64)   # noqa: E731
    masks = [enc.ctx.dropout(torch.ones(dy.shape), 0.25, 3 + (2 << 32), tag) for tag in range(2)]
    dtable, grads = routed_backward(enc, state, dy, balance, masks, values)
    near(enc.dtable, dtable, "table")
    for got, want in zip(enc.grads, grads):
        assert set(got) == set(want)
        for name in want:
            near(got[name], want[name], name)


def test_the_formulas_are_those_of_autograd():
    """The written-out backward pass on rows that are kept as they are."""
    from tests.test_routed_encoder import encoder as plain_encoder, wanted
    enc = plain_encoder()
    ids, dy = batch(5)
    enc.forward(ids, train=True, step=1)
    masks = [enc.ctx.dropout(torch.ones(dy.shape), 0.25, 3 + (1 << 32), tag) for tag in range(2)]
    dtable, grads = routed_backward(enc, enc.state, dy, 0.7, masks, lambda m: m.double())
    _, _, want_table, want = wanted(enc, ids, dy, 1, 0.7)
    near(dtable, want_table, "table")
    for got, of in zip(grads, want):
        for name in of:
            near(got[name], of[name], name)


def test_what_is_kept_in_8_bits_changes_no_row_that_goes_out():
    from paper_2506_22668_amd.encoder import RoutedEncoder
    ids, dy = batch(6)
    args = (NODES, EXPERTS, WIDTH, 40)
    one, other = (RoutedEncoder(PlainPacked(), *args, depth=2, k=K, dtype=torch.float32, p=0.25, seed=3, packed=packed) for packed in (False, True))
    assert torch.equal(one.forward(ids, train=True), other.forward(ids, train=True)) and torch.equal(one.balance, other.balance)
    one.backward(dy)
    other.backward(dy)
    # the last block's biases are sums of gradients that no kept row enters; what the codes are off by (2^-4 of a value) enters the others
    assert torch.equal(one.grads[-1]["b2"], other.grads[-1]["b2"]) and torch.equal(one.grads[-1]["b1"], other.grads[-1]["b1"])
    assert not torch.equal(one.grads[-1]["w2"], other.grads[-1]["w2"]) and not torch.equal(one.grads[-1]["router"], other.grads[-1]["router"])
    assert not torch.equal(one.dtable, other.dtable)
