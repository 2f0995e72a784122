"""The operators of a learned encoder of node features, as measurable cases.

The library explains the answers of a graph network from node features and trained weights. The operators here are what
makes such features and trains their encoder, a residual block per node whose weights depend on the node's type (or on
the expert a router chose): layer norm, products grouped by type with ragged sizes, dropout with the residual sum, and
the groups themselves. Widths are those of the benchmark's models (64 to 512 features, up to the library's widest layer
of 4,096), numbers of rows those of its graphs, from one target's neighbourhood to about a million nodes.
"""
import math

import numpy as np
import torch

own = False

DEV = "cuda:0"
TYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
EPS = 1e-5


def listed():
    return [
        # The rows of one small neighbourhood (33 nodes), normalised for an inference: launch time counts.
        dict(name="norm_small", kind="norm", dtype="f32", rows=33, cols=256, pad=0),
        # All the nodes of a mid-size graph at once.
        dict(name="norm_rows", kind="norm", dtype="bf16", rows=131_072, cols=1024, pad=0),
        # The backward pass of a training step, rows a slice of a wider buffer, with the reduction over all nodes.
        dict(name="norm_grad", kind="norm_bwd", dtype="bf16", rows=100_003, cols=1000, pad=24),
        # The same in fp32 at a width that no vector load divides.
        dict(name="norm_grad_odd", kind="norm_bwd", dtype="f32", rows=30_011, cols=515, pad=0),
        # Dropout of a few odd rows, no residual: the backward form at its smallest.
        dict(name="drop_small", kind="drop", dtype="f16", rows=37, cols=129, pad=0, p=0.5, residual=False),
        # The end of a residual block over all nodes.
        dict(name="drop_residual", kind="drop", dtype="bf16", rows=131_072, cols=1024, pad=0, p=0.1, residual=True),
        # The node types of one neighbourhood ...
        dict(name="groups_small", kind="groups", rows=1_010, groups=8, skew=0.5, loose=0.0),
        # ... and of a graph of a million nodes with nodes of no type.
        dict(name="groups_large", kind="groups", rows=1_000_175, groups=64, skew=0.5, loose=0.02),
        # A handful of nodes, one each type: the weights are what is read.
        dict(name="mm_few_rows", kind="mm", dtype="bf16", rows=8, inner=1024, outer=4096, groups=8, skew=0.0,
             loose=0.0, sorted=False, bias=True, relu=True),
        # The forward product over all the nodes of a graph, types mixed among the rows.
        dict(name="mm_rows", kind="mm", dtype="bf16", rows=131_072, inner=1024, outer=1024, groups=8, skew=0.5,
             loose=0.0, sorted=False, bias=True, relu=True),
        # fp32 weights, as the library's own models have, rows sorted by type, some of no type.
        dict(name="mm_f32", kind="mm", dtype="f32", rows=30_011, inner=512, outer=256, groups=5, skew=0.5, loose=0.02,
             sorted=True, bias=True, relu=False),
        # Both gradients of a training step, types mixed, sizes ragged, the ReLU before it undone in the same pass.
        dict(name="mm_grad", kind="mm_bwd", dtype="bf16", rows=65_521, inner=1024, outer=512, groups=16, skew=0.5,
             loose=0.0, sorted=False, gate=True),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def _width(rng, lo, hi):
    """Half of the widths are multiples of 8 (what models have), half are any."""
    w = _log(rng, lo, hi)
    return w if rng.random() < 0.5 else max(8, w // 8 * 8)


def draw(rng):
    """One more case of the ranges above."""
    kind = rng.choice(["norm", "norm_bwd", "norm_bwd", "drop", "drop", "groups", "mm", "mm", "mm", "mm_bwd", "mm_bwd"])
    dtype = rng.choice(["bf16", "bf16", "f16", "f32"])
    if kind == "groups":
        return dict(kind=kind, rows=_log(rng, 1, 1_000_000), groups=_log(rng, 1, 256), skew=rng.choice([0.0, 0.5, 1.0]),
                    loose=rng.choice([0.0, 0.02]))
    if kind in ("norm", "norm_bwd", "drop"):
        cols = _width(rng, 16, 4096)
        rows = _log(rng, 1, min(400_000, (65_000_000 if dtype == "f32" else 130_000_000) // cols))
        case = dict(kind=kind, dtype=dtype, rows=rows, cols=cols, pad=rng.choice([0, 0, 8, 3]))
        if kind == "drop":
            case.update(p=rng.choice([0.1, 0.3, 0.5]), residual=rng.random() < 0.5)
        return case
    inner, outer = _width(rng, 16, 4096), _width(rng, 16, 4096)
    most = 130_000_000_000 // (inner * outer) // (2 if kind == "mm_bwd" else 1) // (8 if dtype == "f32" else 1)
    # at least one call in three is of a few rows
    rows = rng.randint(1, 64) if rng.random() < 0.33 else _log(rng, 64, max(64, min(400_000, most, 200_000_000 // max(inner, outer))))
    groups = _log(rng, 1, 64)
    groups = max(1, min(groups, 300_000_000 // (inner * outer)))
    case = dict(kind=kind, dtype=dtype, rows=rows, inner=inner, outer=outer, groups=groups,
                skew=rng.choice([0.0, 0.5] if groups > 8 else [0.0, 0.5, 1.0]), loose=rng.choice([0.0, 0.02]),
                sorted=rng.random() < 0.5)
    if kind == "mm":
        case.update(bias=rng.random() < 0.5, relu=rng.random() < 0.5)
    else:
        case.update(gate=rng.random() < 0.5)
    return case


def _normal(g, *shape, dtype=torch.float32, scale=1.0):
    return torch.randn(*shape, generator=g, device=DEV).mul_(scale).to(dtype)


def _rows(g, rows, cols, pad, dtype):
    """Rows with their own mean and spread, `pad` elements apart."""
    x = torch.randn(rows, cols + pad, generator=g, device=DEV)
    x.mul_(0.5 + torch.rand(rows, 1, generator=g, device=DEV)).add_(torch.randn(rows, 1, generator=g, device=DEV))
    return x.to(dtype)[:, :cols]


def _ids(g, case):
    """The group of every row: evenly dealt (skew 0), or with shares that fall off and one group that stays empty; a share
    `loose` of the rows has none."""
    n, m = case["rows"], case["groups"]
    if case["skew"] == 0.0:
        ids = (torch.arange(n, device=DEV) % m)[torch.randperm(n, generator=g, device=DEV)]
    else:
        share = torch.arange(1, m + 1, device=DEV).float().pow(-case["skew"])
        if m >= 4:
            share[1] = 0.0
        ids = torch.searchsorted(torch.cumsum(share / share.sum(), 0), torch.rand(n, generator=g, device=DEV)).clamp_(max=m - 1)
    ids[torch.rand(n, generator=g, device=DEV) < case["loose"]] = -1
    return ids.to(torch.int32)


def _by_group(ids, groups):
    """offsets[g]: rows in the groups before g; order: the rows by group, ascending within each, those of none last."""
    key = torch.where((ids >= 0) & (ids < groups), ids, torch.full_like(ids, groups)).to(torch.int64)
    held, order = torch.sort(key, stable=True)
    return torch.searchsorted(held, torch.arange(groups + 1, device=ids.device)), order.to(torch.int32)


def prepare(case, seed):
    g = torch.Generator(device=DEV)
    g.manual_seed(seed)
    kind, s = case["kind"], dict(case)
    if kind == "groups":
        s["ids"] = _ids(g, case)
        return s
    t = TYPES[case["dtype"]]
    if kind in ("norm", "norm_bwd"):
        s["x"] = _rows(g, case["rows"], case["cols"], case["pad"], t)
        s["weight"], s["bias"] = 1.0 + _normal(g, case["cols"], scale=0.2), _normal(g, case["cols"], scale=0.2)
        if kind == "norm_bwd":
            s["dy"] = _normal(g, case["rows"], case["cols"] + case["pad"], dtype=t)[:, :case["cols"]]
            x = s["x"].double()
            s["mean"] = x.mean(1).float()   # what the forward pass kept
            s["rstd"] = (x.var(1, unbiased=False) + EPS).rsqrt().float()
        return s
    if kind == "drop":
        s["x"] = _normal(g, case["rows"], case["cols"] + case["pad"], dtype=t)[:, :case["cols"]]
        s["residual"] = _normal(g, case["rows"], case["cols"], dtype=t) if case["residual"] else None
        s["seed"] = int(torch.randint(0, 2 ** 62, (1,), generator=g, device=DEV).item())
        return s
    n, k, m, groups = case["rows"], case["inner"], case["outer"], case["groups"]
    ids = _ids(g, case)
    if case["sorted"]:
        ids = torch.sort(torch.where(ids < 0, groups, ids))[0]
    s["offsets"], order = _by_group(ids, groups)
    s["order"] = None if case["sorted"] else order
    sizes = (s["offsets"][1:] - s["offsets"][:-1]).tolist()
    s["most"], s["held"] = max(sizes + [1]), sum(sizes)
    s["x"] = _normal(g, n, k, dtype=t)
    s["w"] = _normal(g, groups, k, m, dtype=t, scale=k ** -0.5)
    if kind == "mm":
        s["bias"] = _normal(g, groups, m, scale=0.5) if case["bias"] else None
    else:
        s["dy"] = _normal(g, n, m, dtype=t)
        if case["gate"]:
            s["x"] = s["x"].clamp_(min=0)   # the output of a ReLU
    return s


def _philox(c0, c1, c2, c3, k0, k1):
    """Philox4x32-10 on int64 tensors that hold 32-bit words."""
    m = 0xFFFFFFFF
    for r in range(10):
        p0, p1 = c0 * 0xD2511F53, c2 * 0xCD9E8D57
        a, b = (k0 + r * 0x9E3779B9) & m, (k1 + r * 0xBB67AE85) & m
        c0, c1, c2, c3 = ((p1 >> 32) & m) ^ c1 ^ a, p1 & m, ((p0 >> 32) & m) ^ c3 ^ b, p0 & m
    return c0, c1, c2, c3


def _kept(rows, cols, p, seed, tag):
    """Element (r, c) is kept where 16 bits are not below round(65536 p): half c % 2 of word c % 8 / 2 of the generator at
    the counter (c / 8, r, tag) under the key `seed`."""
    r = torch.arange(rows, device=DEV)[:, None]
    c = torch.arange((cols + 7) // 8, device=DEV)[None, :]
    zero = torch.zeros_like(r + c)
    words = _philox(zero + c, zero + (r & 0xFFFFFFFF), zero + (r >> 32), zero + tag, seed & 0xFFFFFFFF, seed >> 32)
    halves = torch.stack([h for w in words for h in (w & 0xFFFF, w >> 16)], 2).reshape(rows, -1)[:, :cols]
    return halves >= round(p * 65536)


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
    if kind == "groups":
        return _by_group(s["ids"], s["groups"])
    x = s["x"]
    if kind == "norm":
        v = x.float()
        v = v - v.mean(1, keepdim=True)
        v = v * (v.square().mean(1, keepdim=True) + EPS).rsqrt()
        return (v * s["weight"] + s["bias"]).to(x.dtype)
    if kind == "norm_bwd":
        dy, rstd = s["dy"].float(), s["rstd"][:, None]
        hat = (x.float() - s["mean"][:, None]) * rstd
        g = dy * s["weight"]
        dx = rstd * (g - g.mean(1, keepdim=True) - hat * (g * hat).mean(1, keepdim=True))
        return dx.to(x.dtype), (dy * hat).sum(0), dy.sum(0)
    if kind == "drop":
        t = round(s["p"] * 65536)
        v = torch.where(_kept(s["rows"], s["cols"], s["p"], s["seed"], 1), x.float() * (65536.0 / (65536 - t)), 0.0)
        return (v if s["residual"] is None else s["residual"].float() + v).to(x.dtype)
    w = s["w"].float()
    if kind == "mm":
        xp, place, rows = _padded(s, x)
        y = torch.bmm(xp, w)
        if s["bias"] is not None:
            y = y + s["bias"][:, None]
        if s["relu"]:
            y = torch.relu(y)
        out = torch.zeros(s["rows"], s["outer"], dtype=x.dtype, device=DEV)
        out[rows] = y.view(-1, s["outer"])[place].to(x.dtype)
        return out
    dyp, place, rows = _padded(s, s["dy"])
    xp = _padded(s, x)[0]
    dx = torch.zeros(s["rows"], s["inner"], dtype=x.dtype, device=DEV)
    dx[rows] = torch.bmm(dyp, w.transpose(1, 2).contiguous()).view(-1, s["inner"])[place].to(x.dtype)
    if s["gate"]:
        dx = torch.where(x > 0, dx, 0.0)
    return dx, torch.bmm(xp.transpose(1, 2).contiguous(), dyp).to(s["w"].dtype), dyp.sum(1)


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
    if kind == "groups":
        return ctx.group_rows(s["ids"], s["groups"])
    if kind == "norm":
        return ctx.layer_norm(s["x"], s["weight"], s["bias"], eps=EPS)
    if kind == "norm_bwd":
        return ctx.layer_norm_backward(s["dy"], s["x"], s["mean"], s["rstd"], s["weight"])
    if kind == "drop":
        return ctx.dropout(s["x"], s["p"], s["seed"], tag=1, residual=s["residual"])
    if kind == "mm":
        return ctx.grouped_mm(s["x"], s["w"], s["offsets"], order=s["order"], bias=s["bias"], relu=s["relu"])
    return ctx.grouped_mm_backward(s["dy"], s["x"], s["w"], s["offsets"], order=s["order"],
                                   gate=s["x"] if s["gate"] else None)


def work(case):
    kind, n = case["kind"], case["rows"]
    if kind == "groups":
        return {"bytes": 8.0 * n + 8 * (case["groups"] + 1), "flops": 0.0}
    b = 4 if case["dtype"] == "f32" else 2
    if kind in ("norm", "norm_bwd", "drop"):
        size = float(n) * case["cols"]
        if kind == "norm":
            return {"bytes": 2 * b * size + 8 * case["cols"], "flops": 8 * size}
        if kind == "norm_bwd":
            return {"bytes": 3 * b * size + 8 * n + 12 * case["cols"], "flops": 14 * size}
        return {"bytes": (3 if case["residual"] else 2) * b * size, "flops": (3 if case["residual"] else 2) * size}
    k, m = case["inner"], case["outer"]
    named = 4.0 * n * (not case["sorted"]) + 8 * (case["groups"] + 1)
    if kind == "mm":
        active = min(case["groups"], n)
        return {"bytes": b * (float(n) * (k + m) + float(active) * k * m) + 4 * active * m * case["bias"] + named,
                "flops": 2.0 * n * k * m}
    return {"bytes": b * (float(n) * (2 * k + m) + float(min(case["groups"], n) + case["groups"]) * k * m)
            + 4 * case["groups"] * m + named, "flops": 4.0 * n * k * m}


def _dropped(rows, cols, p, seed, tag):
    """Where dropout leaves nothing, by the generator's definition on numpy's unsigned words."""
    calls, low, half = (cols + 7) // 8, np.uint64(0xFFFFFFFF), np.uint64(32)
    index = np.arange(rows * calls, dtype=np.uint64)
    row, a = np.divmod(index, np.uint64(calls))
    b, c, d = row & low, row >> half, np.full_like(a, tag)
    key = [seed & 0xFFFFFFFF, seed >> 32]
    for _ in range(10):
        left, right = a * np.uint64(0xD2511F53), c * np.uint64(0xCD9E8D57)
        a, c = (right >> half) ^ b ^ np.uint64(key[0]), (left >> half) ^ d ^ np.uint64(key[1])
        b, d = right & low, left & low
        key = [(key[0] + 0x9E3779B9) & 0xFFFFFFFF, (key[1] + 0xBB67AE85) & 0xFFFFFFFF]
    words = np.stack([a, b, c, d], 1).astype(np.uint32)
    halves = words.astype("<u4").view("<u2").reshape(rows, calls * 8)[:, :cols]
    return torch.from_numpy(halves < round(p * 65536)).to(DEV)


def exact(case, seed):
    """The definitions in 64 bits, group by group."""
    kind = case["kind"]
    if kind == "groups":
        return None
    s = prepare(case, seed)
    x = s["x"].double()
    if kind == "norm":
        var, mean = torch.var_mean(x, 1, unbiased=False, keepdim=True)
        return (x - mean) / torch.sqrt(var + EPS) * s["weight"].double() + s["bias"].double()
    if kind == "norm_bwd":
        rstd, dy = s["rstd"].double()[:, None], s["dy"].double()
        hat = (x - s["mean"].double()[:, None]) * rstd
        dhat = dy * s["weight"].double()
        dots = torch.stack([dhat, dhat * hat]).mean(2)
        return (rstd * (dhat - dots[0][:, None] - hat * dots[1][:, None]), torch.einsum("rc,rc->c", dy, hat),
                torch.ones(1, len(dy), dtype=torch.float64, device=DEV).mm(dy)[0])
    if kind == "drop":
        t = round(case["p"] * 65536)
        dropped = _dropped(case["rows"], case["cols"], case["p"], s["seed"], 1)
        out = (x * 65536 / (65536 - t)).masked_fill(dropped, 0.0)
        return out if s["residual"] is None else out + s["residual"].double()
    ends = s["offsets"].tolist()
    out = torch.zeros(case["rows"], case["outer"] if kind == "mm" else case["inner"], dtype=torch.float64, device=DEV)
    dw, db = [], []
    for g in range(case["groups"]):
        at = slice(ends[g], ends[g + 1]) if s["order"] is None else s["order"][ends[g]:ends[g + 1]].long()
        w = s["w"][g].double()
        if kind == "mm":
            y = x[at] @ w if s["bias"] is None else x[at] @ w + s["bias"][g].double()
            out[at] = y.clamp(min=0) if case["relu"] else y
            continue
        dy = s["dy"][at].double()
        out[at] = dy @ w.t()
        dw.append(x[at].t() @ dy)
        db.append(dy.sum(0))
    if kind == "mm":
        return out
    return out.masked_fill(x <= 0, 0.0) if case["gate"] else out, torch.stack(dw), torch.stack(db)
