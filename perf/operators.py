"""The training operators on gathered rows: rows sorted by expert and back with their gradients, and
activations kept in 8 bits with their use in the backward pass.

Every case is one pass through one operator.  Row counts and widths are those of the iterations of the
workloads in ``workload/``: 3 500 rows of 64 values, 76 000 and 177 000 of 128, 820 000 of 256.
"""
from __future__ import annotations

import math

import torch

own = False

TYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
SIZE = {"f32": 4, "bf16": 2, "f16": 2}
BLOCK = 32                      # channels that share a scale
LEAST = -120                    # least exponent of a block
MOST_ROWS, MOST_WIDTH = 820_000, 256


def listed():
    return [
        # Rows sorted by expert.  One row, as a service asks for it: nothing but latency.
        dict(name="sort-one-row", op="sort", rows=1, channels=256, top=2, experts=8, dtype="f32",
             absent=0.0, capacity=0.0),
        # an iteration of the large power-law graph, the features as the gather leaves them
        dict(name="sort-177k", op="sort", rows=177_000, channels=128, top=2, experts=16, dtype="f32",
             absent=0.0, capacity=0.0),
        # And back.  An iteration of the smallest workload, an odd row count and width, padded rows
        # without an expert, experts that take no more than their share
        dict(name="back-3501-odd", op="back", rows=3501, channels=100, top=4, experts=7, dtype="f16",
             absent=0.1, capacity=1.0),
        # the social graph's iteration: the longest there is
        dict(name="back-820k", op="back", rows=820_000, channels=256, top=2, experts=32, dtype="f32",
             absent=0.0, capacity=0.0),
        # The gradients of both.  An ordinary iteration in half the bits
        dict(name="sort-grad-76k", op="sort_grad", rows=76_000, channels=128, top=2, experts=8,
             dtype="bf16", absent=0.0, capacity=1.25),
        # many small experts, eight a row, rows that no vector of 16 bytes divides
        dict(name="sort-grad-41k-odd", op="sort_grad", rows=41_017, channels=250, top=8, experts=128,
             dtype="f32", absent=0.02, capacity=0.0),
        # Activations kept in 8 bits, and restored.  The smallest workload's batch input as it is
        dict(name="keep-3500", op="keep", rows=3500, channels=64, dtype="f32", activation="none"),
        # the longest iteration's pre-activations, and the activation in the same pass
        dict(name="keep-820k-gelu", op="keep", rows=820_000, channels=256, dtype="f32", activation="gelu"),
        # The activation's gradient from the codes.  An ordinary width in half the bits
        dict(name="act-grad-177k", op="act_grad", rows=177_000, channels=256, dtype="bf16",
             activation="silu"),
        # widths that end inside a block, in f16
        dict(name="act-grad-76k-odd", op="act_grad", rows=76_001, channels=333, dtype="f16",
             activation="gelu"),
        # The experts' weight gradients from the codes.  An ordinary iteration, two experts a row
        dict(name="weights-76k", op="weights", rows=76_000, channels=128, out=256, top=2, experts=8,
             dtype="bf16", absent=0.0, capacity=1.25),
        # the longest iteration with gradients as they leave a layer in f32
        dict(name="weights-820k", op="weights", rows=820_000, channels=256, out=256, top=2, experts=32,
             dtype="f32", absent=0.0, capacity=0.0),
    ]


def _log(rng, low, high):
    return int(round(math.exp(rng.uniform(math.log(low), math.log(high)))))


def _width(rng):
    n = _log(rng, 16, 512)
    return n if rng.random() < 0.5 else max(16, n // 8 * 8)


def draw(rng):
    op = rng.choice(["sort", "back", "sort_grad", "keep", "act_grad", "weights"])
    c = dict(op=op, rows=_log(rng, 1, MOST_ROWS), channels=_width(rng), dtype=rng.choice(sorted(TYPES)))
    cost = c["channels"]
    if op in ("keep", "act_grad"):
        c["activation"] = rng.choice(["relu", "silu", "gelu"] if op == "act_grad"
                                     else ["none", "relu", "silu", "gelu"])
    else:
        c["experts"] = _log(rng, 1, 256)
        c["top"] = min(rng.choice([1, 2, 2, 4, 6, 8]), c["experts"])
        c["absent"] = rng.choice([0.0, 0.0, 0.05, 0.3])
        c["capacity"] = rng.choice([0.0, 0.0, 1.0, 1.5])
        if op == "weights":
            c["out"] = _width(rng)
            cost = max(cost, c["out"], math.ceil(c["channels"] * c["out"] / MOST_WIDTH))
        cost *= c["top"]
    c["rows"] = max(1, min(c["rows"], 2 * MOST_ROWS * MOST_WIDTH // cost if "top" in c
                           else MOST_ROWS * MOST_WIDTH // cost))
    return c


def work(case):
    n, C, s = case["rows"], case["channels"], SIZE[case["dtype"]]
    op = case["op"]
    kept = n * (C + -(-C // BLOCK))             # codes and scales
    if op == "keep":
        made = n * C * s * (2 if case["activation"] != "none" else 1)
        return {"bytes": n * C * s + 2 * kept + made, "flops": 4 * n * C}
    if op == "act_grad":
        return {"bytes": kept + 2 * n * C * s, "flops": 8 * n * C}
    p = n * case["top"]
    E = case["experts"]
    rows, slots = n * C * s, p * C * s
    if op == "sort":
        return {"bytes": 8 * p + 8 * p + 8 * (E + 1) + rows + slots, "flops": p}
    if op == "back":
        return {"bytes": 8 * p + slots + rows, "flops": 2 * p * C}
    if op == "sort_grad":
        # dy and z in, dz and dw out; the other gradient's slots in, its rows out
        return {"bytes": 8 * p + rows + 2 * slots + 4 * p + slots + rows, "flops": 4 * p * C}
    D = case["out"]
    return {"bytes": kept + p * D * s + 4 * p + 8 * (E + 1) + 4 * E * C * D, "flops": 2 * p * C * D}


# ---- inputs ------------------------------------------------------------------------------------

def _most(case):
    """Rows an expert takes at most: its share times the capacity factor; None = any number."""
    if not case["capacity"]:
        return None
    return math.ceil(case["rows"] * case["top"] / case["experts"] * case["capacity"])


def _routing(case, gen):
    """What a router leaves: the chosen experts of every row (int64, as a top-k does; -1 for padded rows),
    and their weights.  Some experts are liked more than others."""
    n, E, k = case["rows"], case["experts"], case["top"]
    scores = torch.randn((n, E), generator=gen, device="cuda")
    scores -= 0.5 * torch.log(torch.arange(1, E + 1, device="cuda", dtype=torch.float32))
    best, experts = torch.topk(scores, k, dim=1)
    weights = torch.exp(best - best[:, :1])
    weights /= weights.sum(1, keepdim=True)
    if case["absent"]:
        gone = torch.rand((n, 1), generator=gen, device="cuda") < case["absent"]
        experts = torch.where(gone, torch.full_like(experts, -1), experts)
    return experts, weights


def _codes(x):
    """8-bit blocks of 32 channels: q 2^(e-6), e the exponent of the block's largest magnitude; the scale
    byte is e + 127, or 255 (no number) where a block holds an infinity or a NaN."""
    n, C = x.shape
    blocks = -(-C // BLOCK)
    v = torch.zeros((n, blocks * BLOCK), dtype=torch.float32, device=x.device)
    v[:, :C] = x
    v = v.view(n, blocks, BLOCK)
    fine = torch.isfinite(v).all(2)
    v = torch.where(fine[:, :, None], v, torch.zeros_like(v))
    e = torch.frexp(v.abs().amax(2))[1] - 1
    e = torch.where((v != 0).any(2), e, torch.full_like(e, LEAST)).clamp_(min=LEAST)
    q = torch.round(v * _power(6 - e)[:, :, None]).clamp_(-127, 127).to(torch.int8)
    scales = torch.where(fine, e + 127, torch.full_like(e, 255)).to(torch.uint8)
    return q.view(n, blocks * BLOCK), scales


def _power(e):
    """2^e in f32, exactly, for the exponents of normal numbers."""
    return ((e + 127) << 23).to(torch.int32).view(torch.float32)


def _values(codes, scales, channels):
    n, blocks = scales.shape
    s = scales.to(torch.int32)
    step = torch.where(s == 255, torch.full((), float("nan"), device=codes.device), _power(s - 127 - 6))
    v = codes.view(n, blocks, BLOCK).to(torch.float32) * step[:, :, None]
    return v.view(n, blocks * BLOCK)[:, :channels]


def _normal(gen, shape, dtype, by=1.0):
    return (torch.randn(shape, generator=gen, device="cuda") * by).to(TYPES[dtype])


def _inputs(case, seed):
    gen = torch.Generator(device="cuda")
    gen.manual_seed(seed)
    n, C, op, dtype = case["rows"], case["channels"], case["op"], case["dtype"]
    s = {"case": case}
    if op == "keep":
        s["x"] = _normal(gen, (n, C), dtype)
        return s
    if op == "act_grad":
        s["codes"], s["scales"] = _codes(_normal(gen, (n, C), dtype))
        s["dy"] = _normal(gen, (n, C), dtype, 0.01)
    else:
        experts, s["weights"] = _routing(case, gen)
        p = n * case["top"]
        if op == "sort":
            s["experts"] = experts
            s["x"] = _normal(gen, (n, C), dtype)
            return s
        s["plan"] = _plan(experts, case["experts"], _most(case))
        if op in ("back", "sort_grad"):
            s["z"] = _normal(gen, (p, C), dtype)
        if op == "sort_grad":
            s["dy"] = _normal(gen, (n, C), dtype, 0.01)
            s["g"] = _normal(gen, (p, C), dtype, 0.01)
        if op == "weights":
            s["codes"], s["scales"] = _codes(_normal(gen, (n, C), dtype))
            s["dy"] = _normal(gen, (p, case["out"]), dtype, 0.01)
    return s


def prepare(case, seed):
    """The inputs, and as the program keeps them: the route of the forward pass, the rows it compressed."""
    s = _inputs(case, seed)
    if own:
        import paper_2208_09151_amd as ginex
        if "plan" in s:
            s["route"] = ginex.Route(*s["plan"])
        if "codes" in s:
            s["kept"] = ginex.Compressed(s["codes"], s["scales"], case["channels"])
    return s


# ---- the operators -----------------------------------------------------------------------------

def run(s):
    return _run_own(s) if own else _run_plain(s)


def _run_own(s):
    import paper_2208_09151_amd as ginex
    c, op = s["case"], s["case"]["op"]
    if op == "sort":
        route = ginex.route(s["experts"], c["experts"], capacity=_most(c))
        return {"offsets": route.offsets, "slot": route.slot, "source": route.source,
                "rows": ginex.dispatch(s["x"], route)}
    if op == "back":
        return ginex.combine(s["z"], s["route"], s["weights"])
    if op == "sort_grad":
        dz, dweights = ginex.combine_backward(s["dy"], s["z"], s["route"], s["weights"])
        return {"dz": dz, "dweights": dweights, "dx": ginex.dispatch_backward(s["g"], s["route"])}
    if op == "keep":
        if c["activation"] == "none":
            kept = ginex.compress(s["x"])
            return {"restored": ginex.restore(kept, s["x"].dtype)}
        y, kept = ginex.activate(s["x"], c["activation"])
        return {"y": y, "restored": ginex.restore(kept, s["x"].dtype)}
    if op == "act_grad":
        return ginex.activate_backward(s["kept"], s["dy"], c["activation"])
    return ginex.weight_gradient(s["kept"], s["dy"], s["route"])


def _plan(experts, count, most):
    """offsets of the experts' slots, the slot of every (row, choice) and the row of every slot; slots of an
    expert in the order of the rows, pairs without a slot -1, slots behind the last expert's -1."""
    n, k = experts.shape
    flat = experts.reshape(-1)
    key = torch.where((flat >= 0) & (flat < count), flat, torch.full_like(flat, count))
    key, order = torch.sort(key, stable=True)
    first = torch.searchsorted(key, torch.arange(count + 1, device=key.device))
    sizes = first[1:] - first[:-1]
    if most is not None:
        sizes = sizes.clamp(max=most)
    offsets = torch.zeros(count + 1, dtype=torch.int64, device=key.device)
    torch.cumsum(sizes, 0, out=offsets[1:])
    rank = torch.arange(n * k, device=key.device) - first[key]
    taken = (key < count) & (rank < torch.cat([sizes, sizes.new_zeros(1)])[key])
    place = torch.where(taken, offsets[key] + rank, torch.full_like(rank, -1))
    slot = torch.empty(n * k, dtype=torch.int32, device=key.device)
    slot[order] = place.to(torch.int32)
    source = torch.full((n * k + 1,), -1, dtype=torch.int32, device=key.device)
    source[torch.where(taken, place, torch.full_like(place, n * k))] = (order // k).to(torch.int32)
    return offsets, slot.view(n, k), source[:n * k].contiguous()


def _to_slots(x, source):
    found = x[source.clamp(min=0).long()]
    return torch.where((source >= 0)[:, None], found, torch.zeros_like(found))


def _to_rows(z, slot, weights=None):
    total = None
    for j in range(slot.shape[1]):
        at = slot[:, j]
        part = z[at.clamp(min=0).long()].float()
        if weights is not None:
            part = part * weights[:, j:j + 1]
        part = torch.where((at >= 0)[:, None], part, torch.zeros_like(part))
        total = part if total is None else total + part
    return total


def _activated(x, activation):
    if activation == "relu":
        return torch.where(x < 0, torch.zeros_like(x), x)
    if activation == "silu":
        return x / (1 + torch.exp(-x))
    return 0.5 * x * torch.erfc(-x * math.sqrt(0.5))


def _slope(x, activation):
    """The activation's derivative; no number where x is none."""
    if activation == "relu":
        return torch.where(x > 0, torch.ones_like(x), x * 0)
    if activation == "silu":
        sigma = 1 / (1 + torch.exp(-x))
        return sigma * (1 + x * (1 - sigma))
    return 0.5 * torch.erfc(-x * math.sqrt(0.5)) + x * torch.exp(-0.5 * x * x) / math.sqrt(2 * math.pi)


def _run_plain(s):
    c, op = s["case"], s["case"]["op"]
    if op == "sort":
        offsets, slot, source = _plan(s["experts"], c["experts"], _most(c))
        return {"offsets": offsets, "slot": slot, "source": source, "rows": _to_slots(s["x"], source)}
    if op == "back":
        return _to_rows(s["z"], s["plan"][1], s["weights"]).to(s["z"].dtype)
    if op == "sort_grad":
        _, slot, source = s["plan"]
        dtype, p = s["z"].dtype, source.numel()
        at = torch.where(slot >= 0, slot, torch.full_like(slot, p)).long().reshape(-1)
        of_slot = torch.zeros(p + 1, dtype=torch.float32, device=slot.device)
        of_slot[at] = s["weights"].reshape(-1)
        dz = _to_slots(s["dy"], source).float() * of_slot[:p, None]
        dz = torch.where((source >= 0)[:, None], dz, torch.zeros_like(dz))
        dy = s["dy"].float()
        dots = [(dy * s["z"][slot[:, j].clamp(min=0).long()].float()).sum(1) for j in range(slot.shape[1])]
        dots = torch.stack(dots, 1)
        return {"dz": dz.to(dtype), "dweights": torch.where(slot >= 0, dots, torch.zeros_like(dots)),
                "dx": _to_rows(s["g"], slot).to(dtype)}
    if op == "keep":
        out = {}
        x = s["x"].float()
        if c["activation"] != "none":
            out["y"] = _activated(x, c["activation"]).to(s["x"].dtype)
        codes, scales = _codes(x)
        out["restored"] = _values(codes, scales, c["channels"]).to(s["x"].dtype)
        return out
    x = _values(s["codes"], s["scales"], c["channels"])
    if op == "act_grad":
        return (s["dy"].float() * _slope(x, c["activation"])).to(s["dy"].dtype)
    offsets, _, source = s["plan"]
    x = x[source.clamp(min=0).long()]
    dy = s["dy"].float()
    out = torch.zeros((c["experts"], c["channels"], c["out"]), dtype=torch.float32, device=x.device)
    ends = offsets.tolist()
    for e in range(c["experts"]):
        if ends[e + 1] > ends[e]:
            torch.matmul(x[ends[e]:ends[e + 1]].t(), dy[ends[e]:ends[e + 1]], out=out[e])
    return out


# ---- the definition, in 64 bits ----------------------------------------------------------------

def exact(case, seed):
    s = _inputs(case, seed)
    op = case["op"]
    if op == "sort":
        # a row is copied to every one of its slots; the plan is whole numbers
        x = s["x"].double()
        n, k, E, most = case["rows"], case["top"], case["experts"], _most(case)
        flat = s["experts"].reshape(-1)
        starts, rows = [0], []
        for e in range(E):
            pairs = torch.nonzero(flat == e).flatten()
            pairs = pairs if most is None else pairs[:most]
            rows.append(pairs // k)
            starts.append(starts[-1] + pairs.numel())
        rows = torch.cat(rows)
        out = torch.zeros((n * k, case["channels"]), dtype=torch.float64, device="cuda")
        out[:rows.numel()] = x[rows]
        return {"offsets": None, "slot": None, "source": None, "rows": out}
    if op in ("back", "sort_grad"):
        offsets, slot, source = s["plan"]
        end = int(offsets[-1])
        row = source[:end].long()
        n, k = slot.shape
        # the weight and the place of a slot's pair, from the pairs in slot order
        pairs = torch.nonzero(slot.reshape(-1) >= 0).flatten()
        pairs = pairs[torch.argsort(slot.reshape(-1)[pairs])]
        w = s["weights"].double().reshape(-1)[pairs]
        C = case["channels"]

        def summed(z, by):
            out = torch.zeros((n, C), dtype=torch.float64, device="cuda")
            step = max(1, (1 << 27) // C)
            for lo in range(0, end, step):
                part = z[lo:min(lo + step, end)].double()
                if by is not None:
                    part *= by[lo:lo + step, None]
                out.index_add_(0, row[lo:lo + step], part)
            return out

        if op == "back":
            return summed(s["z"], w)
        dy = s["dy"].double()
        dz = torch.zeros((n * k, C), dtype=torch.float64, device="cuda")
        dz[:end] = dy[row] * w[:, None]
        dots = torch.zeros(n * k, dtype=torch.float64, device="cuda")
        dots[pairs] = (dy[row] * s["z"][:end].double()).sum(1)
        return {"dz": dz, "dweights": dots.view(n, k), "dx": summed(s["g"], None)}
    if op == "keep":
        x = s["x"].double()
        out = {}
        if case["activation"] == "relu":
            out["y"] = x.clamp(min=0)
        elif case["activation"] == "silu":
            out["y"] = x * torch.sigmoid(x)
        elif case["activation"] == "gelu":
            out["y"] = x * torch.special.ndtr(x)
        out["restored"] = torch.empty_like(x)
        for lo in range(0, case["channels"], BLOCK):
            part = x[:, lo:lo + BLOCK]
            top = part.abs().amax(1, keepdim=True)
            step = torch.exp2(torch.floor(torch.log2(top)).clamp(min=LEAST) - 6)
            q = (part / step).round().clamp(-127, 127)
            out["restored"][:, lo:lo + BLOCK] = q * step
        return out
    codes = s["codes"].double()[:, :case["channels"]]
    step = torch.exp2(s["scales"].double() - 133).repeat_interleave(BLOCK, 1)[:, :case["channels"]]
    x = codes * step
    if op == "act_grad":
        if case["activation"] == "relu":
            slope = (x > 0).double()
        elif case["activation"] == "silu":
            sigma = torch.sigmoid(x)
            slope = sigma + x * sigma * (1 - sigma)
        else:
            slope = torch.special.ndtr(x) + x * torch.exp(-x * x / 2) / math.sqrt(2 * math.pi)
        return s["dy"].double() * slope
    offsets, _, source = s["plan"]
    ends = offsets.tolist()
    out = torch.zeros((case["experts"], case["channels"], case["out"]), dtype=torch.float64, device="cuda")
    for e in range(case["experts"]):
        for lo in range(ends[e], ends[e + 1], 1 << 18):
            hi = min(lo + (1 << 18), ends[e + 1])
            out[e] += torch.matmul(x[source[lo:hi].long()].t().contiguous(), s["dy"][lo:hi].double())
    return out
