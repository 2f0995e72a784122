"""The backward pass of RoutedEncoder written out in 64 bits on what its training forward kept: rows that are held in 8 bits stand for what their codes stand for."""
import torch


def routed_backward(enc, state, dy, balance, masks, values):
    """(dtable, a dict of gradients for every block). masks: what dropout multiplies by, one of every block; values: a kept matrix in 64 bits."""
    dy, grads = dy.double(), []
    for (x, y, _, _, w1, w2, router, _, scores, experts, _, counts, _, parts, gain, _), mask in zip(reversed(state.blocks), reversed(masks)):
        x, y, w1, w2, router, gain = x.double(), values(y), w1.double(), w2.double(), router[0].double(), gain.double()
        chosen, n = experts.long(), enc.types
        p = torch.softmax(scores.double(), 1)
        picked = p.gather(1, chosen.t()).t()
        w = picked / picked.sum(0)
        dtotal = mask.double() * dy
        got = dict(w1=torch.zeros_like(w1), b1=dy.new_zeros(n, w1.shape[2]), w2=torch.zeros_like(w2), b2=dy.new_zeros(n, w2.shape[2]))
        dn, dw = torch.zeros_like(x), torch.zeros_like(w)
        for j, (h, out, _, _) in enumerate(parts):
            h, dout = values(h), dtotal * w[j][:, None]
            dw[j] = (dtotal * values(out)).sum(1)
            for e in range(n):
                at = (chosen[j] == e).nonzero()[:, 0]
                dh = (dout[at] @ w2[e].t()) * (h[at] > 0)
                dn[at] += dh @ w1[e].t()
                got["w2"][e] += h[at].t() @ dout[at]
                got["b2"][e] += dout[at].sum(0)
                got["w1"][e] += y[at].t() @ dh
                got["b1"][e] += dh.sum(0)
        # the weights are shares of the chosen, the counts constants of the balance loss
        g = (balance * n * counts[:n].double() / counts[:n].sum().clamp(min=1) / counts[n].clamp(min=1)).expand_as(p)
        g = g.scatter_add(1, chosen.t(), ((dw - (dw * w).sum(0)) / picked.sum(0)).t())
        dscores = p * (g - (p * g).sum(1, keepdim=True))
        got["router"] = y.t() @ dscores
        dn = dn + dscores @ router.t()
        mean = x.mean(1, keepdim=True)
        r = 1 / torch.sqrt((x - mean).square().mean(1, keepdim=True) + 1e-5)
        hat, of = (x - mean) * r, dn * gain
        got["gain"], got["shift"] = (dn * hat).sum(0), dn.sum(0)
        dy = dy + r * (of - of.mean(1, keepdim=True) - hat * (of * hat).mean(1, keepdim=True))
        grads.insert(0, got)
    vocab = enc.table.shape[0]
    there = (state.ids >= 0) & (state.ids < vocab)
    dtable = dy.new_zeros(vocab, dy.shape[1]).index_add_(0, state.ids[there].long(), dy[there] * enc.scale)
    return dtable, grads
