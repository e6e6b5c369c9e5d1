"""Layers of a model on gathered rows: linear layers with their epilogue (also one per expert) and the gradients of
their rows and biases, a whole layer of experts for a few rows, layer norm with its gradients, and the lookup of
learned rows with its gradient.

Every case is one pass through one operator.  Row counts and widths are those of the iterations of the workloads in
``workload/`` (3 500 rows of 64 values, 76 000 and 177 000 of 128, 820 000 of 256) and of the layers behind them.
"""
from __future__ import annotations

import math

import torch

own = False

TYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
SIZE = {"f32": 4, "bf16": 2, "f16": 2}
MOST_ROWS, MOST_WIDTH = 820_000, 256
EPS = 1e-5


def listed():
    return [
        # A linear layer, weights [out, width] as a module has them.  One row, as a service asks for it
        dict(name="linear-one-row", op="linear", rows=1, width=1024, out=1024, dtype="bf16", activation="gelu",
             bias=True, residual=True, turned=True, experts=0),
        # an ordinary iteration in half the bits, a residual block
        dict(name="linear-177k", op="linear", rows=177_000, width=256, out=256, dtype="bf16", activation="gelu",
             bias=True, residual=True, turned=True, experts=0),
        # the longest iteration's first layer, the features as the gather leaves them
        dict(name="linear-820k", op="linear", rows=820_000, width=256, out=256, dtype="f32", activation="relu",
             bias=True, residual=False, turned=True, experts=0),
        # A layer per expert, rows found by the route.  Many small experts, padded rows, odd sizes
        dict(name="experts-9001-odd", op="linear", rows=9001, width=100, out=333, dtype="f16", activation="silu",
             bias=True, residual=False, turned=False, experts=64, top=4, absent=0.1, capacity=1.25),
        # Gradients of rows and biases.  An ordinary iteration, two experts a row
        dict(name="experts-grad-76k", op="linear_grad", rows=76_000, width=128, out=256, dtype="bf16", turned=False,
             experts=8, top=2, absent=0.0, capacity=1.25),
        # the smallest workload's batch through a wide layer, in all bits
        dict(name="linear-grad-3501", op="linear_grad", rows=3501, width=1000, out=250, dtype="f32", turned=True,
             experts=0),
        # A whole layer of experts for few rows.  One row
        dict(name="few-1", op="few", rows=1, width=1024, out=1024, dtype="bf16", activation="silu", bias=False,
             turned=False, experts=64, top=2),
        # a batch of requests, many experts a row, odd sizes
        dict(name="few-48-odd", op="few", rows=48, width=500, out=777, dtype="f16", activation="gelu", bias=True,
             turned=False, experts=32, top=4),
        # Layer norm and its gradients.  Odd rows of the smallest workload
        dict(name="norm-3501-odd", op="norm", rows=3501, width=333, dtype="bf16"),
        # the longest iteration
        dict(name="norm-820k", op="norm", rows=820_000, width=256, dtype="f32"),
        # Lookup of learned rows and its gradient.  A small table in 16 bits, padded ids
        dict(name="lookup-41k-odd", op="lookup", rows=3501, ids=41_017, width=100, dtype="f16", wide=False, absent=0.05),
        # an iteration's neighbours, hubs among them
        dict(name="lookup-1m", op="lookup", rows=177_000, ids=1_000_000, width=128, dtype="f32", wide=True, absent=0.0),
    ]


def _log(rng, low, high):
    return int(round(math.exp(rng.uniform(math.log(low), math.log(high)))))


def _width(rng, most=1024):
    n = _log(rng, 16, most)
    return n if rng.random() < 0.5 else max(16, n // 8 * 8)


def draw(rng):
    op = rng.choice(["linear", "linear", "linear_grad", "few", "norm", "lookup"])
    c = dict(op=op, width=_width(rng), dtype=rng.choice(sorted(TYPES)))
    most = MOST_ROWS * MOST_WIDTH                   # elements of the largest listed rows
    if op == "norm":
        c["width"] = _width(rng, 4096)
        c["rows"] = min(_log(rng, 1, MOST_ROWS), max(1, most // c["width"] - 1))
        return c
    if op == "lookup":
        c["width"] = _width(rng, 512)
        c["rows"] = _log(rng, 1, 177_000)
        c["ids"] = _log(rng, 1, 1_000_000)
        c["ids"] = min(c["ids"], 128_000_000 // c["width"])
        c["rows"] = min(c["rows"], 177_000 * 128 // c["width"])
        c["wide"] = rng.random() < 0.5
        c["absent"] = rng.choice([0.0, 0.0, 0.1, 0.5])
        return c
    c["out"] = _width(rng)
    c["turned"] = rng.random() < 0.5
    if op == "few":
        c["rows"] = _log(rng, 1, 64)
        c["experts"] = _log(rng, 1, 128)
        c["top"] = min(rng.choice([1, 2, 2, 4, 8]), c["experts"])
        c["activation"] = rng.choice(["none", "relu", "silu", "gelu"])
        c["bias"] = rng.random() < 0.5
        return c
    c["experts"] = rng.choice([0, 0, _log(rng, 1, 256)])
    pairs = 1
    if c["experts"]:
        pairs = c["top"] = min(rng.choice([1, 2, 2, 4, 8]), c["experts"])
        c["absent"] = rng.choice([0.0, 0.0, 0.05, 0.3])
        c["capacity"] = rng.choice([0.0, 0.0, 1.0, 1.5])
    if op == "linear":
        c["activation"] = rng.choice(["none", "relu", "silu", "gelu"])
        c["bias"] = rng.random() < 0.6
        c["residual"] = rng.random() < 0.4
    # neither the products nor the bytes of more rows than the largest listed case has
    rows = min(_log(rng, 1, MOST_ROWS), most * MOST_WIDTH // (pairs * (c["width"] + 1) * c["out"]),
               most // (pairs * max(c["width"], c["out"])))
    c["rows"] = max(1, rows)
    return c


def work(case):
    n, C, s, op = case["rows"], case["width"], SIZE[case["dtype"]], case["op"]
    if op == "norm":
        # x in and y out; x and dy in, dx out; the weight and its gradients
        return {"bytes": 5 * n * C * s + 2 * C * s + 8 * C, "flops": 20 * n * C}
    if op == "lookup":
        m = case["ids"]
        # ids, the rows that are there to be found, the found ones; their gradients in and the table's out
        return {"bytes": m * (8 if case["wide"] else 4) + (min(n, m) + m + m + n) * C * s, "flops": 2 * m * C}
    D, E = case["out"], case["experts"]
    if op == "few":
        pairs = n * case["top"]
        chosen = E * (1 - (1 - 1 / E) ** pairs)                 # experts that a row is sent to
        return {"bytes": int(n * (C + D) * s + E * C * s + chosen * C * D * s),
                "flops": 2 * n * E * C + 2 * pairs * C * D}
    p = n * case["top"] if E else n
    weights = max(E, 1) * C * D * s
    plan = 4 * p + 8 * (E + 1) if E else 0
    if op == "linear":
        epilogue = (max(E, 1) * D * s if case["bias"] else 0) + (p * D * s if case["residual"] else 0)
        return {"bytes": n * C * s + weights + plan + epilogue + p * D * s, "flops": 2 * p * C * D}
    return {"bytes": p * D * s + weights + plan + p * C * s + 4 * max(E, 1) * D, "flops": 2 * p * C * D + p * D}


# ---- inputs ------------------------------------------------------------------------------------

def _plan(case, gen):
    """Where a router's choices send the rows: offsets of the experts' slots, the slot of every (row, choice), the row of
    every slot; -1 for padded rows, choices beyond an expert's capacity, and slots behind the last expert's.  Some experts
    are liked more than others."""
    n, E, k = case["rows"], case["experts"], case["top"]
    scores = torch.randn((n, E), generator=gen, device="cuda")
    scores -= 0.5 * torch.log(torch.arange(1, E + 1, device="cuda", dtype=torch.float32))
    experts = torch.topk(scores, k, dim=1)[1]
    if case["absent"]:
        gone = torch.rand((n, 1), generator=gen, device="cuda") < case["absent"]
        experts = torch.where(gone, torch.full_like(experts, E), experts)
    key, order = torch.sort(experts.reshape(-1), stable=True)
    first = torch.searchsorted(key, torch.arange(E + 1, device="cuda"))
    sizes = first[1:] - first[:-1]
    if case["capacity"]:
        sizes = sizes.clamp(max=math.ceil(n * k / E * case["capacity"]))
    offsets = torch.zeros(E + 1, dtype=torch.int64, device="cuda")
    torch.cumsum(sizes, 0, out=offsets[1:])
    rank = torch.arange(n * k, device="cuda") - first[key]
    taken = (key < E) & (rank < torch.cat([sizes, sizes.new_zeros(1)])[key])
    place = torch.where(taken, offsets[key] + rank, torch.full_like(rank, -1))
    slot = torch.empty(n * k, dtype=torch.int32, device="cuda")
    slot[order] = place.to(torch.int32)
    source = torch.full((n * k + 1,), -1, dtype=torch.int32, device="cuda")
    source[torch.where(taken, place, torch.full_like(place, n * k))] = (order // k).to(torch.int32)
    return offsets, slot.view(n, k), source[:n * k].contiguous()


def _normal(gen, shape, dtype, by=1.0):
    return (torch.randn(shape, generator=gen, device="cuda") * by).to(TYPES[dtype])


def _inputs(case, seed):
    gen = torch.Generator(device="cuda")
    gen.manual_seed(seed)
    n, C, op, dtype = case["rows"], case["width"], case["op"], case["dtype"]
    s = {"case": case}
    if op == "norm":
        s["x"] = _normal(gen, (n, C), dtype, 2.0) + 0.5
        s["weight"] = _normal(gen, (C,), dtype, 0.1) + 1
        s["bias"] = _normal(gen, (C,), dtype, 0.1)
        s["dy"] = _normal(gen, (n, C), dtype, 0.01)
        return s
    if op == "lookup":
        # neighbours in a power-law graph: a few rows are asked for again and again
        at = torch.rand(case["ids"], generator=gen, device="cuda", dtype=torch.float64)
        ids = (at ** 3 * n).long().clamp(max=n - 1)
        ids = ids * 7919 % n                        # (hubs are anywhere)
        if case["absent"]:
            gone = torch.rand(case["ids"], generator=gen, device="cuda") < case["absent"]
            ids = torch.where(gone, torch.full_like(ids, -1), ids)
        s["ids"] = ids if case["wide"] else ids.to(torch.int32)
        s["table"] = _normal(gen, (n, C), dtype)
        s["scale"] = math.sqrt(C)
        s["dy"] = _normal(gen, (case["ids"], C), dtype, 0.01)
        return s
    D, E = case["out"], case["experts"]
    shape = (D, C) if case["turned"] else (C, D)
    s["weight"] = _normal(gen, (E, *shape) if E else shape, dtype, 1 / math.sqrt(C))
    if case.get("bias"):
        s["bias"] = _normal(gen, (E, D) if E else (D,), dtype, 0.5)
    if op == "few":
        s["x"] = _normal(gen, (n, C), dtype)
        s["router"] = _normal(gen, (E, C), dtype, 1 / math.sqrt(C))
        return s
    slots = n
    if E:
        s["plan"] = _plan(case, gen)
        slots = n * case["top"]
    if op == "linear":
        s["x"] = _normal(gen, (n, C), dtype)
        if case["residual"]:
            s["residual"] = _normal(gen, (slots, D), dtype)
    else:
        s["dz"] = _normal(gen, (slots, D), dtype, 0.01)
    return s


def prepare(case, seed):
    """The inputs and, as the program keeps it, the route of the rows."""
    s = _inputs(case, seed)
    if own and "plan" in s:
        import paper_2208_09151_amd as ginex
        s["route"] = ginex.Route(*s["plan"])
    return s


# ---- the operators -----------------------------------------------------------------------------

def run(s):
    return _run_own(s) if own else _run_plain(s)


def _activation(c):
    return None if c["activation"] == "none" else c["activation"]


def _run_own(s):
    import paper_2208_09151_amd as ginex
    c, op = s["case"], s["case"]["op"]
    if op == "norm":
        y, stats = ginex.layer_norm(s["x"], s["weight"], s["bias"], eps=EPS, stats=True)
        dx, dweight, dbias = ginex.layer_norm_backward(s["dy"], s["x"], stats, s["weight"])
        return {"y": y, "dx": dx, "dweight": dweight, "dbias": dbias}
    if op == "lookup":
        return {"rows": ginex.lookup(s["table"], s["ids"], scale=s["scale"]),
                "dtable": ginex.lookup_backward(s["dy"], s["ids"], c["rows"], scale=s["scale"])}
    weight = s["weight"].mT if c["turned"] else s["weight"]
    if op == "few":
        return ginex.expert_layer(s["x"], s["router"], weight, c["top"], activation=_activation(c), bias=s.get("bias"))
    if op == "linear":
        return ginex.linear(s["x"], weight, bias=s.get("bias"), activation=_activation(c), residual=s.get("residual"),
                            route=s.get("route"))
    return {"drows": ginex.linear_backward(s["dz"], weight, route=s.get("route")),
            "dbias": ginex.bias_gradient(s["dz"], route=s.get("route"))}


def _activated(x, activation):
    if activation == "none":
        return x
    if activation == "relu":
        return torch.where(x < 0, torch.zeros_like(x), x)
    if activation == "silu":
        return x / (1 + torch.exp(-x))
    return 0.5 * x * torch.erfc(-x * math.sqrt(0.5))


def _product(x, weight, turned):
    return x @ (weight.t() if turned else weight)


def _run_plain(s):
    c, op, dtype = s["case"], s["case"]["op"], TYPES[s["case"]["dtype"]]
    if op == "norm":
        x, weight, bias, dy = (s[k].float() for k in ("x", "weight", "bias", "dy"))
        centred = x - x.mean(1, keepdim=True)
        rstd = 1 / torch.sqrt((centred * centred).mean(1, keepdim=True) + EPS)
        unit = centred * rstd
        y = unit * weight + bias
        a = dy * weight
        dx = rstd * (a - a.mean(1, keepdim=True) - unit * (a * unit).mean(1, keepdim=True))
        return {"y": y.to(dtype), "dx": dx.to(dtype), "dweight": (dy * unit).sum(0), "dbias": dy.sum(0)}
    if op == "lookup":
        ids, table = s["ids"].long(), s["table"]
        there = (ids >= 0)[:, None]
        found = table[ids.clamp(min=0)].float() * s["scale"]
        grad = torch.where(there, s["dy"].float(), torch.zeros((), device=ids.device))
        dtable = torch.zeros(table.shape, dtype=torch.float32, device=ids.device)
        dtable.index_add_(0, ids.clamp(min=0), grad)
        return {"rows": torch.where(there, found, torch.zeros_like(found)).to(dtype),
                "dtable": (dtable * s["scale"]).to(dtype)}
    weight = s["weight"].float()
    if op == "few":
        x = s["x"].float()
        # (in 64 bits: which experts are chosen may hang on the last bits of their scores)
        scores, order = torch.sort(s["x"].double() @ s["router"].double().t(), dim=1, descending=True, stable=True)
        top = c["top"]
        p = torch.exp(scores[:, :top] - scores[:, :1])
        p = (p / p.sum(1, keepdim=True)).float()
        chosen = order[:, :top]
        y = torch.zeros((c["rows"], c["out"]), dtype=torch.float32, device=x.device)
        for e in torch.unique(chosen).tolist():
            row, j = torch.nonzero(chosen == e, as_tuple=True)
            z = _product(x[row], weight[e], c["turned"])
            if "bias" in s:
                z = z + s["bias"][e].float()
            y.index_add_(0, row, p[row, j][:, None] * _activated(z, c["activation"]))
        return y.to(dtype)
    experts = c["experts"]
    if experts:
        offsets, _, source = s["plan"]
        ends = offsets.tolist()
    if op == "linear":
        x = s["x"].float()
        if not experts:
            z = _product(x, weight, c["turned"])
            if "bias" in s:
                z = z + s["bias"].float()
            y = _activated(z, c["activation"])
            return (y + s["residual"].float() if "residual" in s else y).to(dtype)
        out = torch.zeros((source.numel(), c["out"]), dtype=torch.float32, device=x.device)
        for e in range(experts):
            lo, hi = ends[e], ends[e + 1]
            if hi > lo:
                z = _product(x[source[lo:hi].long()], weight[e], c["turned"])
                if "bias" in s:
                    z = z + s["bias"][e].float()
                out[lo:hi] = _activated(z, c["activation"])
                if "residual" in s:
                    out[lo:hi] += s["residual"][lo:hi].float()
        return out.to(dtype)
    dz = s["dz"].float()
    if not experts:
        return {"drows": _product(dz, weight, not c["turned"]).to(dtype), "dbias": dz.sum(0)}
    drows = torch.zeros((dz.shape[0], c["width"]), dtype=torch.float32, device=dz.device)
    dbias = torch.zeros((experts, c["out"]), dtype=torch.float32, device=dz.device)
    for e in range(experts):
        lo, hi = ends[e], ends[e + 1]
        if hi > lo:
            drows[lo:hi] = _product(dz[lo:hi], weight[e], not c["turned"])
            dbias[e] = dz[lo:hi].sum(0)
    return {"drows": drows.to(dtype), "dbias": dbias}


# ---- the definition, in 64 bits ----------------------------------------------------------------

STEP = 1 << 17                  # rows at a time


def _exact_activation(x, activation):
    if activation == "relu":
        return x.clamp(min=0)
    if activation == "silu":
        return x * torch.sigmoid(x)
    if activation == "gelu":
        return x * torch.special.ndtr(x)
    return x


def exact(case, seed):
    s = _inputs(case, seed)
    op, n, C = case["op"], case["rows"], case["width"]
    if op == "norm":
        weight, bias = s["weight"].double(), s["bias"].double()
        y = torch.empty((n, C), dtype=torch.float64, device="cuda")
        dx = torch.empty_like(y)
        dweight = torch.zeros(C, dtype=torch.float64, device="cuda")
        dbias = torch.zeros_like(dweight)
        for lo in range(0, n, STEP):
            x, dy = s["x"][lo:lo + STEP].double(), s["dy"][lo:lo + STEP].double()
            variance, mean = torch.var_mean(x, 1, keepdim=True, correction=0)
            spread = torch.sqrt(variance + EPS)
            unit = (x - mean) / spread
            y[lo:lo + STEP] = torch.addcmul(bias, unit, weight)
            a = dy * weight
            # (I - 1 1^T / C - unit unit^T / C) a / spread
            dx[lo:lo + STEP] = (a - (a.sum(1, keepdim=True) + unit * (a * unit).sum(1, keepdim=True)) / C) / spread
            dweight += (dy * unit).sum(0)
            dbias += dy.sum(0)
        return {"y": y, "dx": dx, "dweight": dweight, "dbias": dbias}
    if op == "lookup":
        ids = s["ids"].long()
        at = torch.nonzero(ids >= 0).flatten()
        rows = torch.zeros((case["ids"], C), dtype=torch.float64, device="cuda")
        dtable = torch.zeros((n, C), dtype=torch.float64, device="cuda")
        for lo in range(0, at.numel(), STEP):
            part = at[lo:lo + STEP]
            rows[part] = s["table"][ids[part]].double() * s["scale"]
            dtable.index_add_(0, ids[part], s["dy"][part].double() * s["scale"])
        return {"rows": rows, "dtable": dtable}
    weight = s["weight"].double()
    if case["turned"]:
        weight = weight.transpose(-1, -2).contiguous()          # [.., width, out]
    D, E = case["out"], case["experts"]
    bias = s["bias"].double() if "bias" in s else torch.zeros((E, D) if E else (D,), dtype=torch.float64, device="cuda")
    if op == "few":
        x = s["x"].double()
        best, chosen = torch.topk(torch.mm(x, s["router"].double().t().contiguous()), case["top"], dim=1)
        share = torch.zeros((n, E), dtype=torch.float64, device="cuda").scatter_(1, chosen, torch.softmax(best, 1))
        y = torch.zeros((n, D), dtype=torch.float64, device="cuda")
        for e in range(E):
            if bool((share[:, e] > 0).any()):
                y += share[:, e:e + 1] * _exact_activation(torch.addmm(bias[e], x, weight[e]), case["activation"])
        return y
    slots = n * case["top"] if E else n
    spans = [(0, 0, n)]
    source = None
    if E:
        offsets, _, source = s["plan"]
        ends = offsets.tolist()
        spans = [(e, ends[e], ends[e + 1]) for e in range(E)]
    else:
        weight, bias = weight[None], bias[None]
    cut = [(e, lo, min(lo + STEP, b)) for e, a, b in spans for lo in range(a, b, STEP)]
    if op == "linear":
        y = torch.zeros((slots, D), dtype=torch.float64, device="cuda")
        for e, lo, hi in cut:
            x = s["x"][lo:hi] if source is None else s["x"].index_select(0, source[lo:hi])
            y[lo:hi] = _exact_activation(torch.addmm(bias[e], x.double(), weight[e]), case["activation"])
            if "residual" in s:
                y[lo:hi] += s["residual"][lo:hi].double()
        return y
    drows = torch.zeros((slots, C), dtype=torch.float64, device="cuda")
    dbias = torch.zeros((max(E, 1), D), dtype=torch.float64, device="cuda")
    for e, lo, hi in cut:
        dz = s["dz"][lo:hi].double()
        drows[lo:hi] = torch.mm(dz, weight[e].t().contiguous())
        dbias[e] += torch.mm(torch.ones((1, hi - lo), dtype=torch.float64, device="cuda"), dz)[0]
    return {"drows": drows, "dbias": dbias if E else dbias[0]}
