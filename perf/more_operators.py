"""The operators of an encoder that learns its nodes' features, their experts and keeps little of it, as measurable cases.

The library's encoder works on rows of features whose group (a type) is given. The operators here are what it lacks to learn both from
a bare graph, and to train over many nodes: rows looked up in a table by the node's id, with the table's gradient; a router that
chooses every row's experts from its scores, counts them and says how evenly they are used, with its gradient; and activations that are
kept for the backward pass in 8 bits, with the gradients of the products by group that read them. Widths are those of the benchmark's models (64 to
512 features, up to the library's widest layer), numbers of rows those of its graphs, from one target's neighbourhood to about a million nodes.
"""
import math

import numpy as np
import torch

own = False

DEV = "cuda:0"
TYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
BYTES = {"f32": 4, "bf16": 2, "f16": 2}
BLOCK = 32   # columns that share a scale


def listed():
    return [
        # The nodes of one small neighbourhood looked up for an inference: launch time counts.
        dict(name="embed_small", kind="embed", dtype="f32", table="f32", rows=33, cols=256, vocab=2_000, skew=0.0, loose=0.0, scale=1.0),
        # The nodes of a training step out of an fp32 table, rows for products in bf16; nodes of many edges come up often.
        dict(name="embed_rows", kind="embed", dtype="bf16", table="f32", rows=262_144, cols=512, vocab=100_003, skew=0.75, loose=0.0, scale=16.0),
        # The table's gradient over one neighbourhood.
        dict(name="embed_grad_small", kind="embed_bwd", dtype="f32", table="f32", rows=1_010, cols=64, vocab=2_000, skew=0.5, loose=0.0, scale=1.0),
        # A million lookups, a few ids of which take a large share, some of none: a table's row is a sum of 1 to 90,000 rows.
        dict(name="embed_grad", kind="embed_bwd", dtype="bf16", table="f32", rows=1_000_175, cols=128, vocab=50_021, skew=1.0, loose=0.02, scale=8.0),
        # A table much larger than the step, of a width that no vector load divides: what is written is mostly zeros.
        dict(name="embed_grad_wide", kind="embed_bwd", dtype="f16", table="f16", rows=30_011, cols=515, vocab=200_003, skew=0.0, loose=0.0, scale=1.0),
        # One neighbourhood's rows to one of eight experts each.
        dict(name="route_small", kind="route", dtype="f32", rows=33, experts=8, k=1, renorm=False, closed=0.0, padded=0.0),
        # All the nodes of a graph of a million to two of 64 experts each.
        dict(name="route_rows", kind="route", dtype="bf16", rows=1_000_175, experts=64, k=2, renorm=True, closed=0.0, padded=0.0),
        # Many experts, an odd number, some closed to some rows, rows of padding without any.
        dict(name="route_odd", kind="route", dtype="f32", rows=30_011, experts=515, k=8, renorm=False, closed=0.1, padded=0.05),
        # The scores' gradient in a training step, from the weights' and the balance loss'.
        dict(name="route_grad", kind="route_bwd", dtype="bf16", rows=131_072, experts=256, k=4, renorm=True, closed=0.0, padded=0.02),
        # Activations of all nodes into 8 bits and back.
        dict(name="pack_rows", kind="pack", dtype="bf16", rows=131_072, cols=1024, pad=0, spread=1.0),
        # Both gradients of products over a few rows, from kept activations: the weights are what is read and written.
        dict(name="packed_grad_few", kind="packed", dtype="bf16", rows=64, inner=1024, outer=1024, groups=8, skew=0.0, loose=0.0, sorted=False, gate=True),
        # The same in a training step over many, types mixed, the kept rows those behind a ReLU, which is undone in the same pass.
        dict(name="packed_grad", kind="packed", dtype="bf16", rows=65_521, inner=1024, outer=512, groups=16, skew=0.5, loose=0.0, sorted=False, gate=True),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def _width(rng, lo, hi):
    """Half of the widths are multiples of 8 (what models have), half are any."""
    w = _log(rng, lo, hi)
    return w if rng.random() < 0.5 else max(8, w // 8 * 8)


def draw(rng):
    """One more case of the ranges above."""
    kind = rng.choice(["embed", "embed_bwd", "embed_bwd", "route", "route", "route_bwd", "pack", "packed", "packed"])
    dtype = rng.choice(["bf16", "bf16", "f16", "f32"])
    most = 65_000_000 if dtype == "f32" else 130_000_000   # elements
    if kind in ("embed", "embed_bwd"):
        cols = _width(rng, 8, 2048)
        table = "f32" if rng.random() < 0.5 else dtype
        return dict(kind=kind, dtype=dtype, table=table, cols=cols, rows=_log(rng, 1, min(1_000_000, most // cols)),
                    vocab=_log(rng, 1, min(1_000_000, 60_000_000 // cols)), skew=rng.choice([0.0, 0.5, 1.0]), loose=rng.choice([0.0, 0.02]),
                    scale=rng.choice([1.0, 8.0]))
    if kind in ("route", "route_bwd"):
        experts = _log(rng, 2, 1024)
        return dict(kind=kind, dtype=dtype, experts=experts, rows=_log(rng, 1, min(1_000_000, most // 2 // experts)), k=rng.randint(1, min(8, experts)),
                    renorm=rng.random() < 0.5, closed=rng.choice([0.0, 0.0, 0.1]), padded=rng.choice([0.0, 0.05]))
    if kind == "pack":
        cols = _width(rng, 16, 4096)
        return dict(kind=kind, dtype=dtype, cols=cols, rows=_log(rng, 1, min(400_000, most // cols)), pad=rng.choice([0, 0, 8, 3]),
                    spread=rng.choice([1.0, 3.0]))
    inner, outer = _width(rng, 16, 2048), _width(rng, 16, 2048)
    work = 34_000_000_000 // (inner * outer) // (8 if dtype == "f32" else 1)
    rows = rng.randint(1, 64) if rng.random() < 0.33 else _log(rng, 64, max(64, min(400_000, work, 100_000_000 // max(inner, outer))))
    groups = max(1, min(_log(rng, 1, 64), 100_000_000 // (inner * outer)))
    return dict(kind=kind, dtype=dtype, rows=rows, inner=inner, outer=outer, groups=groups, skew=rng.choice([0.0, 0.5]), loose=rng.choice([0.0, 0.02]),
                sorted=rng.random() < 0.5, gate=rng.random() < 0.7)


def _normal(g, *shape, dtype=torch.float32, scale=1.0):
    return torch.randn(*shape, generator=g, device=DEV).mul_(scale).to(dtype)


def _chosen(g, n, m, skew, loose):
    """n ids of m: evenly drawn (skew 0) or with shares that fall off by their rank, the ranks spread over the ids; a share `loose` is -1."""
    share = torch.arange(1, m + 1, device=DEV, dtype=torch.float64).pow(-skew)
    ids = torch.searchsorted(torch.cumsum(share / share.sum(), 0), torch.rand(n, generator=g, device=DEV, dtype=torch.float64)).clamp_(max=m - 1)
    ids = torch.randperm(m, generator=g, device=DEV)[ids]
    ids[torch.rand(n, generator=g, device=DEV) < loose] = -1
    return ids.to(torch.int32)


def _scores(g, case):
    """A router's scores: experts that differ in how much they are liked, some closed to some rows (-inf), rows of padding closed to all."""
    n, e = case["rows"], case["experts"]
    x = torch.randn(n, e, generator=g, device=DEV).add_(_normal(g, e, scale=0.5))
    if case["closed"]:
        x[torch.rand(n, e, generator=g, device=DEV) < case["closed"]] = -math.inf
    if case["padded"]:
        x[torch.rand(n, generator=g, device=DEV) < case["padded"]] = -math.inf
    return x.to(TYPES[case["dtype"]])


def prepare(case, seed):
    g = torch.Generator(device=DEV)
    g.manual_seed(seed)
    kind, s = case["kind"], dict(case)
    t = TYPES[case["dtype"]]
    if kind in ("embed", "embed_bwd"):
        s["ids"] = _chosen(g, case["rows"], case["vocab"], case["skew"], case["loose"])
        if kind == "embed":
            s["weights"] = _normal(g, case["vocab"], case["cols"], dtype=TYPES[case["table"]])
        else:
            s["dy"] = _normal(g, case["rows"], case["cols"], dtype=t)
        return s
    if kind in ("route", "route_bwd"):
        s["x"] = _scores(g, case)
        if kind == "route_bwd":   # what the forward pass left, and the gradients that came back
            s["ids"], _, s["counts"], _, s["lse"] = _route(s["x"], case["k"], case["renorm"])
            s["dweights"] = _normal(g, case["k"], case["rows"])
            s["dloss"] = _normal(g, 1)[0] * 100.0
        return s
    if kind == "pack":
        x = torch.randn(case["rows"], case["cols"] + case["pad"], generator=g, device=DEV)
        x.mul_(torch.exp(_normal(g, case["rows"], 1, scale=case["spread"])))
        s["x"] = x.to(t)[:, :case["cols"]]
        return s
    n, k, m, groups = case["rows"], case["inner"], case["outer"], case["groups"]
    ids = _chosen(g, n, groups, case["skew"], case["loose"])
    key = torch.where(ids < 0, groups, ids).to(torch.int64)
    held, order = torch.sort(key, stable=True)
    s["offsets"], s["order"] = torch.searchsorted(held, torch.arange(groups + 1, device=DEV)), None if case["sorted"] else order.to(torch.int32)
    sizes = (s["offsets"][1:] - s["offsets"][:-1]).tolist()
    s["most"], s["held"] = max(sizes + [1]), sum(sizes)
    x = _normal(g, n, k, dtype=t)
    s["codes"], s["scales"] = _pack(x.clamp_(min=0) if case["gate"] else x)
    s["w"], s["dy"] = _normal(g, groups, k, m, dtype=t, scale=k ** -0.5), _normal(g, n, m, dtype=t)
    return s


# ---- the plain forms ----------------------------------------------------------------------------------------------------------------------


def _route(x, k, renorm):
    """(ids int32[k, rows], weights[k, rows], counts int64[experts + 1], loss, lse[rows]): the k highest scores of a row, ties to the lowest
    expert, those of -inf left out (-1, weight 0); their probabilities (renorm: over their sum); how often each expert was chosen, and the rows that
    have one; experts * sum over experts of (share of the choices) * (mean probability over these rows)."""
    v, (n, e) = x.float(), x.shape
    most = v.amax(1, keepdim=True)
    some = most > -math.inf
    top = torch.where(some, most, 0.0)
    q = torch.exp(v - top)
    total = q.sum(1, keepdim=True)
    p = q / torch.where(some, total, 1.0)
    lse = torch.where(some, top + torch.log(total), -math.inf)[:, 0]
    left, order, ids = v.clone(), torch.arange(e, device=x.device), []
    for _ in range(k):
        most = left.amax(1, keepdim=True)
        first = torch.where(left == most, order, e).amin(1)
        ids.append(torch.where(most[:, 0] > -math.inf, first, -1))
        left.scatter_(1, first[:, None], -math.inf)
    ids = torch.stack(ids)
    weights = torch.where(ids >= 0, p.gather(1, ids.clamp(min=0).t()).t(), 0.0)
    if renorm:
        weights = weights / torch.where(some[:, 0], weights.sum(0), 1.0)
    chosen = torch.bincount((ids + 1).reshape(-1), minlength=e + 1)[1:]
    rows = some.sum()
    share = chosen.double() / chosen.sum().clamp(min=1)
    loss = e * (share * p.sum(0, dtype=torch.float64)).sum() / rows.clamp(min=1)
    return ids.to(torch.int32), weights, torch.cat([chosen, rows[None]]), loss.float(), lse


def _route_grad(s):
    x, ids, counts = s["x"].float(), s["ids"].long(), s["counts"]
    e = x.shape[1]
    some = s["lse"] > -math.inf
    p = torch.where(some[:, None], torch.exp(x - torch.where(some, s["lse"], 0.0)[:, None]), 0.0)
    chosen = ids >= 0
    dw = torch.where(chosen, s["dweights"], 0.0)
    at = ids.clamp(min=0).t()
    if s["renorm"]:
        weights = torch.where(chosen, p.gather(1, at).t(), 0.0)
        total = torch.where(some, weights.sum(0), 1.0)
        dw = torch.where(chosen, (dw - (dw * weights).sum(0) / total) / total, 0.0)
    share = counts[:e].double() / counts[:e].sum().clamp(min=1) / counts[e].clamp(min=1)
    g = (s["dloss"].double() * e * share).float().expand_as(p).clone().scatter_add_(1, at, dw.t())
    return (p * (g - (p * g).sum(1, keepdim=True))).to(s["x"].dtype)


def _power(e):
    """2^e in 32 bits, e from -126 to 127 (ldexp goes through pow, whose last bit is not sure)."""
    return ((e + 127) << 23).to(torch.int32).view(torch.float32)


def _pack(x):
    """(codes e4m3[rows, cols], scales uint8[rows, blocks of 32 columns]) with x ~ codes * 2^(scales - 127): the scale is the smallest power of two
    that leaves a block's finite values at or below 448, codes are the nearest values (to even), but no value that is not 0 becomes 0, none
    passes the largest one of x's type, and infinities become NaN."""
    rows, cols = x.shape
    v = torch.nn.functional.pad(x.float(), (0, -cols % BLOCK)).view(rows, -1, BLOCK)
    fine = torch.isfinite(v)
    bits = torch.where(fine, v.abs(), 0.0).amax(2).view(torch.int32)
    high, wide = bits >> 23, (bits & 0x7FFFFF) > 0x600000
    scale = torch.where(bits == 0, 127, (high - 8 + wide.int()).clamp(min=1))
    top = torch.where(wide & (high == (142 if x.dtype == torch.float16 else 254)), 240.0, 448.0)[:, :, None]
    q = v * _power(127 - scale[:, :, None])
    least = 2.0 ** -9
    q = torch.where((q.abs() < least) & (v != 0), torch.where(v < 0, -least, least), torch.minimum(torch.maximum(q, -top), top))
    codes = torch.where(fine, q, math.nan).to(torch.float8_e4m3fn).view(rows, -1)[:, :cols].contiguous()
    return codes, scale.to(torch.uint8)


def _unpack(codes, scales):
    cols = codes.shape[1]
    return codes.float() * _power(scales.int().sub_(127)).repeat_interleave(BLOCK, 1)[:, :cols]


def _padded(s, a):
    """The rows of `a` by group, [groups, most, width] in 32 bits, and the places of the rows in it."""
    pos = torch.arange(s["held"], device=DEV)
    group = torch.searchsorted(s["offsets"][1:], pos, right=True)
    place = group * s["most"] + pos - s["offsets"][group]
    rows = pos if s["order"] is None else s["order"][:s["held"]].long()
    out = torch.zeros(s["groups"] * s["most"], a.shape[1], device=DEV)
    out[place] = a[rows].float()
    return out.view(s["groups"], s["most"], -1), place, rows


def _plain(s):
    kind = s["kind"]
    if kind in ("embed", "embed_bwd"):
        ids = s["ids"].long()
        there = (ids >= 0) & (ids < s["vocab"])
        at = torch.where(there, ids, 0)
        if kind == "embed":
            return torch.where(there[:, None], s["weights"][at].float() * s["scale"], 0.0).to(TYPES[s["dtype"]])
        held, order = torch.sort(torch.where(there, ids, s["vocab"]), stable=True)
        ends = torch.searchsorted(held, torch.arange(s["vocab"] + 1, device=DEV))
        upto = torch.nn.functional.pad(s["dy"].t().double()[:, order].cumsum(1), (1, 0))   # (sums of up to all rows)
        return ((upto[:, ends[1:]] - upto[:, ends[:-1]]) * s["scale"]).t().contiguous().to(TYPES[s["table"]])
    if kind == "route":
        return _route(s["x"], s["k"], s["renorm"])
    if kind == "route_bwd":
        return _route_grad(s)
    if kind == "pack":
        return _unpack(*_pack(s["x"])).to(s["x"].dtype)
    t, x = s["w"].dtype, _unpack(s["codes"], s["scales"])
    dyp, place, rows = _padded(s, s["dy"])
    xp = _padded(s, x)[0]
    dx = torch.zeros(s["rows"], s["inner"], dtype=t, device=DEV)
    dx[rows] = torch.bmm(dyp, s["w"].float().transpose(1, 2).contiguous()).view(-1, s["inner"])[place].to(t)
    if s["gate"]:
        dx = torch.where(x > 0, dx, 0.0)
    return dx, torch.bmm(xp.transpose(1, 2).contiguous(), dyp).to(t), dyp.sum(1)


# ---- the calls ------------------------------------------------------------------------------------------------------------------------------

_context = None


def _ctx():
    """The one handle of a user's program."""
    global _context
    if _context is None:
        from paper_2506_22668_amd import Context
        _context = Context(DEV)
    return _context


def run(state):
    s = state
    if not own:
        return _plain(s)
    ctx, kind = _ctx(), s["kind"]
    if kind == "embed":
        return ctx.embed(s["weights"], s["ids"], scale=s["scale"], dtype=TYPES[s["dtype"]])
    if kind == "embed_bwd":
        return ctx.embed_backward(s["dy"], s["ids"], s["vocab"], scale=s["scale"], dtype=TYPES[s["table"]])
    if kind == "route":
        return ctx.route(s["x"], s["k"], renorm=s["renorm"])
    if kind == "route_bwd":
        return ctx.route_backward(s["x"], s["lse"], s["ids"], s["counts"], dweights=s["dweights"], dloss=s["dloss"], renorm=s["renorm"])
    if kind == "pack":
        return ctx.unpack_rows(ctx.pack_rows(s["x"]), s["x"].dtype)
    from paper_2506_22668_amd import Packed
    x = Packed(s["codes"], s["scales"])
    return ctx.grouped_mm_backward(s["dy"], x, s["w"], s["offsets"], order=s["order"], gate=x if s["gate"] else None)


def _distinct(case):
    """The different ids among a case's lookups, on average."""
    share = np.arange(1, case["vocab"] + 1, dtype=np.float64) ** -case["skew"]
    return float(-np.expm1(case["rows"] * (1 - case["loose"]) * np.log1p(-np.minimum(share / share.sum(), 1 - 1e-12))).sum())


def work(case):
    kind, n, b = case["kind"], float(case["rows"]), BYTES[case["dtype"]]
    if kind == "embed":
        return {"bytes": 4 * n + b * n * case["cols"] + BYTES[case["table"]] * _distinct(case) * case["cols"], "flops": n * case["cols"]}
    if kind == "embed_bwd":
        return {"bytes": 4 * n + b * n * (1 - case["loose"]) * case["cols"] + float(BYTES[case["table"]]) * case["vocab"] * case["cols"], "flops": n * case["cols"]}
    if kind == "route":
        size = n * case["experts"]
        return {"bytes": b * size + n * (8 * case["k"] + 4) + 8 * (case["experts"] + 1), "flops": (5 + case["k"]) * size}
    if kind == "route_bwd":
        size = n * case["experts"]
        return {"bytes": 2 * b * size + n * (8 * case["k"] + 4) + 8 * (case["experts"] + 1), "flops": 6 * size}
    if kind == "pack":
        return {"bytes": 2 * b * n * case["cols"], "flops": 4 * n * case["cols"]}
    k, m, groups = case["inner"], case["outer"], case["groups"]
    kept = n * (k + (k + BLOCK - 1) // BLOCK)
    return {"bytes": kept + b * n * (k + m) + b * float(min(groups, n) + groups) * k * m + 4.0 * groups * m + 4 * n * (not case["sorted"]) + 8 * (groups + 1),
            "flops": 4 * n * k * m}


# ---- the definitions in 64 bits ---------------------------------------------------------------------------------------------------------------


def _exact_route(x, k, renorm):
    held, at = torch.sort(x.double(), dim=1, descending=True, stable=True)
    n, e = x.shape
    lse = torch.logsumexp(held, 1)
    have = torch.isfinite(held[:, :k])
    prob = torch.exp(held - torch.where(torch.isfinite(lse), lse, 0.0)[:, None])
    ids, weights = at[:, :k].masked_fill(~have, -1), prob[:, :k].masked_fill(~have, 0.0)
    if renorm:
        weights = torch.nan_to_num(weights / weights.sum(1, keepdim=True), nan=0.0)
    rows = torch.isfinite(lse).sum()
    mean = torch.zeros(e, dtype=torch.float64, device=x.device).index_add_(0, at.reshape(-1), prob.reshape(-1)) / max(int(rows), 1)
    counts = (ids.reshape(-1)[:, None] == torch.arange(e, device=x.device)).sum(0) if n * k * e < 1 << 28 else \
        torch.histc(ids[have].double(), e, -0.5, e - 0.5).long()
    loss = e * torch.dot(counts.double(), mean) / max(int(counts.sum()), 1)
    return ids.t().to(torch.int32), weights.t(), torch.cat([counts, rows.view(1)]), loss, lse


def exact(case, seed):
    kind = case["kind"]
    s = prepare(case, seed)
    if kind == "embed":
        ids = s["ids"].long()
        table = torch.cat([s["weights"].double() * case["scale"], torch.zeros(1, case["cols"], dtype=torch.float64, device=DEV)])
        return table.index_select(0, torch.where((ids < 0) | (ids >= case["vocab"]), case["vocab"], ids))
    if kind == "embed_bwd":
        out = torch.zeros(case["vocab"], case["cols"], dtype=torch.float64, device=DEV)
        known = (s["ids"] >= 0).nonzero()[:, 0]
        return out.index_add_(0, s["ids"][known].long(), s["dy"][known].double()).mul_(case["scale"])
    if kind == "route":
        return _exact_route(s["x"], case["k"], case["renorm"])
    if kind == "route_bwd":
        x, e = s["x"].double(), case["experts"]
        z = torch.where(torch.isfinite(x.amax(1, keepdim=True)), x, 0.0)
        p = torch.softmax(z, 1) * torch.isfinite(x.amax(1, keepdim=True))
        took = torch.zeros_like(p)
        dw = torch.zeros_like(p)
        for j in range(case["k"]):
            hit = (s["ids"][j][:, None] == torch.arange(e, device=DEV)).double()
            took += hit
            dw += hit * s["dweights"][j].double()[:, None]
        if case["renorm"]:   # w = q / sum(q) over the chosen, q = p there
            total = (p * took).sum(1, keepdim=True)
            total = torch.where(total > 0, total, 1.0)
            dw = took * (dw / total - (dw * p).sum(1, keepdim=True) / total.square())
        n_rows, n_chosen = max(int(s["counts"][e]), 1), max(int(s["counts"][:e].sum()), 1)
        g = dw + s["dloss"].double() * e / (float(n_rows) * n_chosen) * s["counts"][:e].double()
        return p * g - p * (p * g).sum(1, keepdim=True)
    if kind == "pack":
        x = s["x"].double()
        cols, half = case["cols"], case["dtype"] == "f16"
        two = lambda e: ((e.long() + 1023) << 52).view(torch.float64)   # noqa: E731
        out = torch.empty_like(x)
        for c in range(0, cols, BLOCK):
            v = x[:, c:c + BLOCK]
            most = v.abs().amax(1, keepdim=True)
            part, power = torch.frexp(most)   # most = part * 2^power, part in [1/2, 1)
            unit = two(torch.where(most > 0, torch.where(part > 0.875, power - 8, power - 9), 0).clamp(min=-126))
            q = v / unit
            step = two(torch.frexp(q.abs().clamp(min=2.0 ** -6))[1] - 4)
            near = torch.round(q / step) * step
            near = torch.where((near == 0) & (v != 0), torch.sign(v) * 2.0 ** -9, near)
            near = torch.where(near.abs() * unit > (65504.0 if half else 3.4e38), torch.sign(v) * 240.0, near)
            out[:, c:c + BLOCK] = near * unit
        return out
    k, m = case["inner"], case["outer"]
    ends = s["offsets"].tolist()
    grid = s["codes"].double().view(case["rows"], -1) * ((s["scales"].long() + (1023 - 127)) << 52).view(torch.float64).repeat_interleave(BLOCK, 1)[:, :k]
    dx = torch.zeros(case["rows"], k, dtype=torch.float64, device=DEV)
    dw, db = [], []
    for g in range(case["groups"]):
        at = slice(ends[g], ends[g + 1]) if s["order"] is None else s["order"][ends[g]:ends[g + 1]].long()
        dy = s["dy"][at].double()
        dx[at] = dy @ s["w"][g].double().t()
        dw.append(grid[at].t() @ dy)
        db.append(dy.sum(0))
    return dx.masked_fill(grid <= 0, 0.0) if case["gate"] else dx, torch.stack(dw), torch.stack(db)
