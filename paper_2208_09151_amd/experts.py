"""A layer of experts on gathered rows, and a small training run over it: sampling, changesets, the feature
cache and the gather in front, the training operators behind.

  python -m paper_2208_09151_amd.experts [--config 1] [--steps 40] [--blocks 0]

``ExpertLayer`` sends every row to the experts its router likes best, one linear layer and an activation
each, and adds their answers up by the router's weights.  What the backward pass needs of the rows and of
the activations' inputs is kept in 8 bits (8.25 with the scales, instead of 32): the rows once, not once per
expert, as the weight gradient looks them up by the route.  The experts' answers are kept as they are, for the
gradient of the router's weights.  The products of forward pass and input gradient are torch's, an expert at a
time, and need the experts' sizes on the host: the layer waits for the GPU once and cannot be captured into a
graph.  ``ExpertLayer.answer`` is its form for a few rows, without gradients and without a wait.

``Block`` is a residual block with a layer of experts inside whose products are ``linear``'s, which looks rows up by the route
and waits for nothing.
"""
from __future__ import annotations

import argparse
import math
import os
import sys

import torch

from .layers import expert_layer, layer_norm, linear, lookup, lookup_backward
from .training import (Activation, Combine, Compressed, Route, _first_derivative, activate, combine,  # noqa: F401
                       compress, dispatch, dispatch_backward, route, weight_gradient)

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


def _spans(ends):
    """(expert, first slot, last slot + 1) of the experts that have rows."""
    return [(e, a, b) for e, (a, b) in enumerate(zip(ends[:-1], ends[1:])) if b > a]


class ExpertLinear(torch.autograd.Function):
    """Rows to their slots and through their expert's weights [experts, width, out].  Keeps the rows in 8
    bits for the weight gradient."""

    @staticmethod
    def forward(ctx, x, weight, r, ends):
        rows = dispatch(x, r)
        out = torch.empty((rows.shape[0], weight.shape[2]), dtype=x.dtype, device=x.device)
        for e, a, b in _spans(ends):
            torch.mm(rows[a:b], weight[e], out=out[a:b])
        out[ends[-1]:].zero_()
        kept = compress(x)
        ctx.width, ctx.ends = kept.width, ends
        ctx.save_for_backward(weight, kept.codes, kept.scales, *r._tensors())
        return out

    @staticmethod
    @_first_derivative
    def backward(ctx, grad):
        weight, codes, scales, *route = ctx.saved_tensors
        r = Route(*route)
        grad = grad.contiguous()
        dx = dw = None
        if ctx.needs_input_grad[1]:
            dw = weight_gradient(Compressed(codes, scales, ctx.width), grad, r).to(weight.dtype)
        if ctx.needs_input_grad[0]:
            drows = torch.empty((grad.shape[0], weight.shape[1]), dtype=grad.dtype, device=grad.device)
            for e, a, b in _spans(ctx.ends):
                torch.mm(grad[a:b], weight[e].t(), out=drows[a:b])
            dx = dispatch_backward(drows, r)
        return dx, dw, None, None


class ExpertLayer(torch.nn.Module):
    """``top`` of ``experts`` linear layers with an activation ("relu", "silu", "gelu") for every row.
    ``capacity``: rows an expert takes at most, as a multiple of its even share; rows beyond it do without."""

    def __init__(self, width, out, experts, top=2, activation="gelu", capacity=None):
        super().__init__()
        self.experts, self.top, self.activation, self.capacity = experts, top, activation, capacity
        self.router = torch.nn.Linear(width, experts, bias=False)
        self.weight = torch.nn.Parameter(torch.randn(experts, width, out) / math.sqrt(width))

    def forward(self, x):
        best, chosen = torch.topk(self.router(x).float(), self.top, dim=1)
        weights = torch.softmax(best, dim=1)
        most = None if self.capacity is None else \
            math.ceil(x.shape[0] * self.top / self.experts * self.capacity)
        r = route(chosen, self.experts, capacity=most)
        ends = r.offsets.tolist()           # (the products need them on the host)
        y, _ = activate(ExpertLinear.apply(x, self.weight, r, ends), self.activation)
        return combine(y, r, weights)


    @torch.no_grad()
    def answer(self, x):
        """The layer for up to 64 rows, in two launches; no expert is ever full."""
        return expert_layer(x, self.router.weight, self.weight, self.top, self.activation)


class Block(torch.nn.Module):
    """x + down(experts(norm(x))): layer norm, ``top`` of ``experts`` linear layers with a bias and an activation, their sum by
    the router's weights, and a linear layer back to ``width`` with x as its residual."""

    def __init__(self, width, hidden, experts, top=2, activation="gelu"):
        super().__init__()
        self.experts, self.top, self.activation = experts, top, activation
        self.norm_weight = torch.nn.Parameter(torch.ones(width))
        self.norm_bias = torch.nn.Parameter(torch.zeros(width))
        self.router = torch.nn.Linear(width, experts, bias=False)
        self.up = torch.nn.Parameter(torch.randn(experts, width, hidden) / math.sqrt(width))
        self.up_bias = torch.nn.Parameter(torch.zeros(experts, hidden))
        self.down = torch.nn.Linear(hidden, width)

    def forward(self, x):
        n = layer_norm(x, self.norm_weight, self.norm_bias)
        best, chosen = torch.topk(self.router(n).float(), self.top, dim=1)
        r = route(chosen, self.experts)
        h = linear(n, self.up, self.up_bias, self.activation, route=r)
        h = combine(h, r, torch.softmax(best, dim=1))
        return linear(h, self.down.weight.t(), self.down.bias, residual=x)

    @torch.no_grad()
    def answer(self, x):
        """The block for up to 64 rows."""
        n = layer_norm(x, self.norm_weight, self.norm_bias)
        h = expert_layer(n, self.router.weight, self.up, self.top, self.activation, self.up_bias)
        return linear(h, self.down.weight.t(), self.down.bias, residual=x)


class SumOfRows(torch.autograd.Function):
    """out[s] = the sum of the rows r with of[r] = s: what lookup's gradient does, and lookup is its gradient."""

    @staticmethod
    def forward(ctx, rows, of, sums):
        ctx.save_for_backward(of)
        return lookup_backward(rows, of, sums)

    @staticmethod
    @_first_derivative
    def backward(ctx, grad):
        return lookup(grad.contiguous(), *ctx.saved_tensors), None, None


class Classifier(torch.nn.Module):
    """An expert layer on all sampled rows, ``blocks`` residual blocks, the mean over a seed's first-hop neighbours, and a linear
    head."""

    def __init__(self, width, hidden, classes, experts, blocks=0):
        super().__init__()
        self.layer = ExpertLayer(width, hidden, experts, capacity=2.0)
        self.head = torch.nn.Linear(2 * hidden, classes)
        self.blocks = torch.nn.ModuleList(Block(hidden, 2 * hidden, experts) for _ in range(blocks))

    def forward(self, x, rowptr, col):
        h = self.layer(x)
        for block in self.blocks:
            h = block(h)
        seeds = rowptr.numel() - 1
        count = (rowptr[1:] - rowptr[:-1])
        of = torch.repeat_interleave(torch.arange(seeds, device=x.device), count)
        if len(self.blocks):                # (these add up in one order, both ways)
            around = SumOfRows.apply(lookup(h, col), of, seeds)
        else:
            around = torch.zeros((seeds, h.shape[1]), dtype=h.dtype, device=x.device).index_add(0, of, h[col.long()])
        around = around / count.clamp(min=1)[:, None]
        return self.head(torch.cat([h[:seeds], around], 1))


def train(config=1, steps=40, hidden=64, experts=8, classes=8, rate=0.02, report=print, blocks=0):
    """Trains the classifier on the batches of a synthetic workload, one superbatch after the other; the
    label of a node is its largest feature of the first ``classes``.  Returns the losses."""
    import paper_2208_09151_amd as ginex
    if ROOT not in sys.path:
        sys.path.insert(0, ROOT)
    from workload import make_workload
    from workload.configs import seed_batches, train_nodes

    w = make_workload(config, device="cuda")
    cfg = w.cfg
    cache = ginex.FeatureCache(w.features, cfg.cap)
    nodes = train_nodes(cfg.num_nodes, cfg.train_frac, cfg.seed, "cuda")
    with torch.random.fork_rng(devices=[]):
        torch.random.default_generator.manual_seed(0)       # (torch.manual_seed would seed the GPU's, too)
        model = Classifier(cfg.feat_dim, hidden, classes, experts, blocks).cuda()
    adam = torch.optim.Adam(model.parameters(), lr=rate)
    losses = []
    while len(losses) < steps:
        first = len(losses)
        seeds, so = seed_batches(nodes, cfg.batch, cfg.S, cfg.seed, first)
        sampled = ginex.sample_superbatch(w.offsets, w.indices, seeds.cuda(), so.numpy(), cfg.fanout,
                                          first_batch_index=first)
        cs = ginex.changeset(cfg.num_nodes, sampled.ids, sampled.ids_offsets, cfg.cap)
        cache.init(cs.init_ids)
        io, co = sampled.ids_offsets, cs.cs_offsets
        for i in range(min(cfg.S, steps - first)):
            at, ch = slice(io[i], io[i + 1]), slice(co[i], co[i + 1])
            x = cache.gather(sampled.ids[at], None, cs.in_ids[ch], cs.out_ids[ch], cs.in_positions[ch],
                             src_line=cs.src_line[at], n_slow=int(cs.miss_count[i]))
            rowptr, col = sampled.adj_segment(i, 0)
            labels = x[:rowptr.numel() - 1, :classes].argmax(1)
            loss = torch.nn.functional.cross_entropy(model(x, rowptr, col), labels)
            adam.zero_grad()
            loss.backward()
            adam.step()
            losses.append(float(loss.detach()))
            if report and (len(losses) % 10 == 0 or len(losses) == 1):
                report(f"step {len(losses)}: {x.shape[0]} rows, loss {losses[-1]:.3f}")
    return losses


def main():
    ap = argparse.ArgumentParser(description=__doc__.split("\n\n")[0])
    ap.add_argument("--config", type=int, default=1)
    ap.add_argument("--steps", type=int, default=40)
    ap.add_argument("--hidden", type=int, default=64)
    ap.add_argument("--experts", type=int, default=8)
    ap.add_argument("--blocks", type=int, default=0)
    args = ap.parse_args()
    losses = train(args.config, args.steps, args.hidden, args.experts, blocks=args.blocks)
    print(f"loss {losses[0]:.3f} -> {losses[-1]:.3f} in {len(losses)} steps")


if __name__ == "__main__":
    main()
