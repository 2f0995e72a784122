"""A learned encoder of node features: residual blocks whose weights depend on the node's type.

    h = x + dropout(relu(norm(x) W1[type] + b1[type]) W2[type] + b2[type])

The block runs on the library's operators on rows (`Context.layer_norm`, `group_rows`, `grouped_mm`, `dropout` and their
gradients); what it puts out is what `Context.set_features` takes. Run as a program it trains a small encoder on nodes of three types,
hands the features to a GCN and explains one of its answers:

    python -m paper_2506_22668_amd.encoder
"""
import torch


class TypedEncoder:
    """`depth` residual blocks over rows of `width` features of `types` kinds. Parameters are fp32; products run in `dtype`
    (fp32, bf16 or fp16). `forward(..., train=True)` keeps what `backward` needs; `update` is a step of plain gradient descent."""

    def __init__(self, ctx, types, width, hidden, depth=1, dtype=torch.bfloat16, p=0.1, seed=0):
        g = torch.Generator(device=ctx.device)
        g.manual_seed(seed)
        self.ctx, self.types, self.dtype, self.p, self.seed = ctx, types, dtype, p, seed
        normal = lambda *shape, scale: torch.randn(*shape, generator=g, device=ctx.device) * scale   # noqa: E731
        zeros = lambda *shape: torch.zeros(*shape, device=ctx.device)   # noqa: E731
        self.blocks = [dict(gain=zeros(width) + 1, shift=zeros(width), w1=normal(types, width, hidden, scale=width ** -0.5), b1=zeros(types, hidden),
                            w2=normal(types, hidden, width, scale=hidden ** -0.5), b2=zeros(types, width)) for _ in range(depth)]
        self._kept, self.grads = [], []

    def forward(self, x, node_type, train=False, step=0):
        """Rows of x through the blocks, in `dtype`. node_type: int32, one a row (a row of no type passes through unchanged). The
        dropout of a training step is a function of (seed, step, block, row, column)."""
        c = self.ctx
        offsets, order = c.group_rows(node_type, self.types)
        x, self._kept = x.to(self.dtype), []
        for tag, b in enumerate(self.blocks):
            w1, w2 = b["w1"].to(self.dtype), b["w2"].to(self.dtype)
            y, mean, rstd = c.layer_norm(x, b["gain"], b["shift"], want_stats=True)
            h = c.grouped_mm(y, w1, offsets, order=order, bias=b["b1"], relu=True)
            out = c.grouped_mm(h, w2, offsets, order=order, bias=b["b2"])
            if train:
                self._kept.append((x, y, h, mean, rstd, w1, w2, offsets, order, self.seed + (step << 32), tag))
            x = c.dropout(out, self.p if train else 0.0, self.seed + (step << 32), tag, residual=x)
        return x

    def backward(self, dy):
        """The gradient of the rows that went in; those of the parameters are left in `grads`, one dict a block."""
        c, self.grads = self.ctx, []
        dy = dy.to(self.dtype)
        for b, (x, y, h, mean, rstd, w1, w2, offsets, order, seed, tag) in zip(reversed(self.blocks), reversed(self._kept)):
            dout = c.dropout(dy, self.p, seed, tag)
            dh, dw2, db2 = c.grouped_mm_backward(dout, h, w2, offsets, order=order, gate=h)
            dn, dw1, db1 = c.grouped_mm_backward(dh, y, w1, offsets, order=order)
            dx, dgain, dshift = c.layer_norm_backward(dn, x, mean, rstd, b["gain"])
            dy = dy + dx
            self.grads.insert(0, dict(gain=dgain, shift=dshift, w1=dw1, b1=db1, w2=dw2, b2=db2))
        return dy

    def update(self, rate):
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
