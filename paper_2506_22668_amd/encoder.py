"""A learned encoder of node features: residual blocks whose weights depend on the node's type.

    h = x + dropout(relu(norm(x) W1[type] + b1[type]) W2[type] + b2[type])

The block runs on the library's operators on rows (`Context.layer_norm`, `group_rows`, `grouped_mm`, `dropout` and their
gradients); what it puts out is what `Context.set_features` takes. Run as a program it trains a small encoder on nodes of three types,
hands the features to a GCN and explains one of its answers:

    python -m paper_2506_22668_amd.encoder
"""
import torch

from .binding import DS_EINVAL, DistShapError


class _State:
    """What a backward pass reads of its training forward."""

    def __init__(self, p, seed):
        self.p, self.seed, self.shape, self.blocks, self._held = p, seed, None, [], []

    def hold(self, *tensors):
        """Tensors that are read where they lie: their values have to be the same at the backward pass. (Inference tensors do not count their changes.)"""
        self._held += [(t, t._version) for t in tensors if not t.is_inference()]

    def changed(self):
        return any(t._version != version for t, version in self._held)


class TypedEncoder:
    """`depth` residual blocks over rows of `width` features of `types` kinds. Parameters are fp32; products run in `dtype`
    (fp32, bf16 or fp16). `forward(..., train=True)` leaves what `backward` needs in `state`; `update` is a step of plain gradient descent."""

    def __init__(self, ctx, types, width, hidden, depth=1, dtype=torch.bfloat16, p=0.1, seed=0):
        g = torch.Generator(device=ctx.device)
        g.manual_seed(seed)
        self.ctx, self.types, self.dtype, self.p, self.seed = ctx, types, dtype, p, seed
        normal = lambda *shape, scale: torch.randn(*shape, generator=g, device=ctx.device) * scale   # noqa: E731
        zeros = lambda *shape: torch.zeros(*shape, device=ctx.device)   # noqa: E731
        self.blocks = [dict(gain=zeros(width) + 1, shift=zeros(width), w1=normal(types, width, hidden, scale=width ** -0.5), b1=zeros(types, hidden),
                            w2=normal(types, hidden, width, scale=hidden ** -0.5), b2=zeros(types, width)) for _ in range(depth)]
        self.state, self.grads = None, []
        self._waiting = 0   # training forwards since the last backward pass

    @property
    def _kept(self):
        return self.state.blocks if self.state else []

    def forward(self, x, node_type, train=False, step=0):
        """Rows of x through the blocks, in `dtype`. node_type: int32, one a row (a row of no type passes through unchanged). The
        dropout of a training step is a function of (seed, step, block, row, column). An evaluation (train=False) leaves `state` alone; the
        parameters of a training step, and x where it is of `dtype` already, stay as they are until its backward pass."""
        c = self.ctx
        offsets, order = c.group_rows(node_type, self.types)
        state = _State(self.p, self.seed + (step << 32))
        rows, x = x, x.to(self.dtype)
        state.shape = x.shape
        if train and x is rows:
            state.hold(x)
        for tag, b in enumerate(self.blocks):
            w1, w2 = b["w1"].to(self.dtype), b["w2"].to(self.dtype)
            y, mean, rstd = c.layer_norm(x, b["gain"], b["shift"], want_stats=True)
            h = c.grouped_mm(y, w1, offsets, order=order, bias=b["b1"], relu=True)
            out = c.grouped_mm(h, w2, offsets, order=order, bias=b["b2"])
            if train:
                state.blocks.append((x, y, h, mean, rstd, w1, w2, offsets, order, b["gain"], tag))
                state.hold(b["gain"], *(w for w in (w1, w2) if w is b["w1"] or w is b["w2"]))
            x = c.dropout(out, self.p if train else 0.0, state.seed, tag, residual=x)
        if train:
            self.state = state
            self._waiting += 1
        return x

    def backward(self, dy, state=None):
        """The gradient of the rows that went in; those of the parameters are left in `grads`, one dict a block. `state`: what `self.state` was
        after the forward that dy belongs to; it can be left out where there was one training forward since the last backward pass."""
        c, self.grads = self.ctx, []
        if state is None:
            if self._waiting != 1:
                raise DistShapError(DS_EINVAL, "backward without a training forward of its own" if self._waiting == 0 else
                                    f"{self._waiting} training forwards wait for a backward pass: give the `state` of the one that is meant")
            state = self.state
        if state.shape != dy.shape:
            raise DistShapError(DS_EINVAL, f"dy has shape {tuple(dy.shape)}, {tuple(state.shape)} went out")
        if state.changed():
            raise DistShapError(DS_EINVAL, "the rows or the parameters of this forward have been changed since")
        dy, grads = dy.to(self.dtype), []
        for x, y, h, mean, rstd, w1, w2, offsets, order, gain, tag in reversed(state.blocks):
            dout = c.dropout(dy, state.p, state.seed, tag)
            dh, dw2, db2 = c.grouped_mm_backward(dout, h, w2, offsets, order=order, gate=h)
            dn, dw1, db1 = c.grouped_mm_backward(dh, y, w1, offsets, order=order)
            dx, dgain, dshift = c.layer_norm_backward(dn, x, mean, rstd, gain)
            dy = dy + dx
            grads.insert(0, dict(gain=dgain, shift=dshift, w1=dw1, b1=db1, w2=dw2, b2=db2))
        self.grads, self._waiting = grads, 0
        return dy

    def update(self, rate):
        if len(self.grads) != len(self.blocks):
            raise DistShapError(DS_EINVAL, "update without the gradients of a backward pass")
        for b, g in zip(self.blocks, self.grads):
            for name, v in b.items():
                v.sub_(rate * g[name].float())


def main(nodes=2000, width=64, steps=60):
    from . import Context
    ctx = Context("cuda:0")
    g = torch.Generator(device="cuda:0")
    g.manual_seed(1)
    rand = lambda *shape: torch.randn(*shape, generator=g, device="cuda:0")   # noqa: E731
    kind = torch.randint(0, 3, (nodes,), generator=g, device="cuda:0").to(torch.int32)
    x, target = rand(nodes, width), torch.zeros(nodes, width, device="cuda:0")
    for k, turn in enumerate(rand(3, width, width) * width ** -0.5):   # every type has a map of its own to learn
        target[kind == k] = x[kind == k] @ turn
    enc = TypedEncoder(ctx, 3, width, 2 * width, depth=2)
    for step in range(steps):
        out = enc.forward(x, kind, train=True, step=step)
        off = out.float() - target
        if step % 10 == 0 or step == steps - 1:
            print(f"step {step}: mean squared error {off.square().mean().item():.4f}", flush=True)
        enc.backward(off * (2.0 / nodes))
        enc.update(0.02)
    # a ring with chords, a GCN on the learned features, and the edges that one of its answers rests on
    near = torch.tensor([-7, -1, 1, 7])
    col = ((torch.arange(nodes)[:, None] + near) % nodes).sort(1)[0].reshape(-1).to(torch.int32)
    ctx.set_graph(torch.arange(nodes + 1) * 4, col)
    ctx.set_features(enc.forward(x, kind).float())
    ctx.set_gcn([rand(width, 32) * 0.2, rand(32, 4) * 0.2])
    phi, src, dst, report, _ = ctx.explain(5, 4096, seed=3)
    top = phi.abs().topk(3)[1]
    print(f"node 5 is of class {report.pred_class}; of {report.num_players} edges, these weigh most:",
          [(int(src[i]), int(dst[i]), round(float(phi[i]), 4)) for i in top])
    ctx.close()


if __name__ == "__main__":
    main()
