"""include/ginex_layers.h: every entry point is exported and bound, and refuses what it cannot do before anything is
launched (no GPU)."""
import ctypes as C
import os
import re

import pytest

from paper_2208_09151_amd import _lib

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
FAKE = 0x10000                  # never read: every call here fails on the host


def error():
    return _lib.load().ginex_last_error().decode()


def rows(n=10, width=64, stride=None, kind=0, data=FAKE):
    return _lib.RowsDesc(data, n, width, width if stride is None else stride, kind)


def routing(n=10, top=2, experts=4, offsets=FAKE, slot=FAKE, source=FAKE):
    return _lib.RoutingDesc(n, top, experts, offsets, slot, source)


def weights(experts=4, turned=0, width=64, out=32, stride=None, expert_stride=None, kind=0, data=FAKE):
    return _lib.WeightsDesc(data, experts, turned, width, out, (width if turned else out) if stride is None else stride,
                            width * out if expert_stride is None else expert_stride, kind)


def codes(n=20, width=32, data=FAKE, scales=FAKE):
    return _lib.CodesDesc(n, width, data, scales)


def ref(x):
    return None if x is None else C.byref(x)


def test_every_declared_symbol_is_exported_and_bound():
    text = open(os.path.join(ROOT, "include", "ginex_layers.h")).read()
    text = re.sub(r"/\*.*?\*/", "", text, flags=re.S)
    names = sorted(set(re.findall(r"\b(ginex_[a-z_]+)\s*\(", text)))
    assert sorted(_lib.LAYER_SIGNATURES) == names and len(names) == 11
    for n in names:
        assert getattr(_lib.load(), n) is not None


def test_constants_of_the_binding_are_the_headers():
    from paper_2208_09151_amd import layers
    text = open(os.path.join(ROOT, "include", "ginex_layers.h")).read()
    value = {k: int(v) for k, v in re.findall(r"#define GINEX_(\w+) (\d+)", text)}
    assert (layers.FEW_ROWS, layers.FEW_TOP) == (value["MAX_FEW_ROWS"], value["MAX_FEW_TOP"])


BAD_ROWS = [(rows(kind=3), "type"), (rows(width=0), "width"), (rows(width=(1 << 20) + 1), "width"), (rows(stride=63), "stride"),
            (rows(data=None), "null"), (rows(data=FAKE + 2), "aligned"), (rows(n=-1), "rows")]


@pytest.mark.parametrize("bad, says", BAD_ROWS)
def test_rows_that_no_call_takes(bad, says):
    lib, good, big = _lib.load(), rows(), 1 << 40
    w, r = weights(1), rows(20, 32)
    assert lib.ginex_linear(ref(bad), ref(w), None, 0, None, None, 0, ref(r), None, None) == -1 and says in error()
    assert lib.ginex_linear(ref(good), ref(w), None, 0, None, None, 0, ref(bad), None, None) == -1 and says in error()
    assert lib.ginex_linear(ref(good), ref(w), None, 0, ref(bad), None, 0, ref(rows(10, 32)), None, None) == -1
    assert says in error()
    assert lib.ginex_bias_gradient(ref(bad), None, FAKE, FAKE, big, None) == -1 and says in error()
    assert lib.ginex_expert_layer(ref(bad), ref(rows(4)), ref(weights()), None, 2, 0, ref(rows(10, 32)), FAKE, big, None) == -1
    assert says in error()
    assert lib.ginex_expert_layer(ref(good), ref(bad), ref(weights()), None, 2, 0, ref(rows(10, 32)), FAKE, big, None) == -1
    assert says in error()
    assert lib.ginex_layer_norm(ref(bad), None, None, 1e-5, ref(good), None, None) == -1 and says in error()
    assert lib.ginex_layer_norm_backward(ref(bad), ref(good), FAKE, None, ref(good), FAKE, FAKE, FAKE, big, None) == -1
    assert lib.ginex_layer_norm_backward(ref(good), ref(good), FAKE, None, ref(bad), FAKE, FAKE, FAKE, big, None) == -1
    assert lib.ginex_lookup(ref(bad), FAKE, 0, 1.0, ref(good), None) == -1 and says in error()
    assert lib.ginex_lookup_backward(ref(bad), FAKE, 0, 1.0, ref(good), FAKE, big, None) == -1 and says in error()


@pytest.mark.parametrize("bad, says", [
    (weights(0), "experts"), (weights(1025), "experts"), (weights(turned=2), "turned"), (weights(width=0), "width"),
    (weights(out=(1 << 20) + 1), "out"), (weights(stride=31), "stride"), (weights(turned=1, stride=63), "stride"),
    (weights(expert_stride=-1), "expert_stride"), (weights(data=None), "null"), (weights(data=FAKE + 1), "aligned"),
    (weights(kind=7), "type"), (None, "null")])
def test_weights_that_no_call_takes(bad, says):
    lib = _lib.load()
    assert lib.ginex_linear(ref(rows()), ref(bad), None, 0, None, ref(routing()), 0, ref(rows(20, 32)), None, None) == -1
    assert says in error()
    assert lib.ginex_expert_layer(ref(rows()), ref(rows(4)), ref(bad), None, 2, 0, ref(rows(10, 32)), FAKE, 1 << 40, None) == -1
    assert says in error()


def test_linear_refusals():
    lib = _lib.load()

    def call(x=rows(), w=weights(), bias=None, act=0, res=None, r=routing(), by_slot=0, y=rows(20, 32), kept=None):
        return lib.ginex_linear(ref(x), ref(w), bias, act, ref(res), ref(r), by_slot, ref(y), ref(kept), None)

    assert call(x=rows(kind=1)) == -1 and "type" in error()
    assert call(y=rows(20, 32, kind=2)) == -1 and "type" in error()
    assert call(x=rows(width=65)) == -1 and "wide" in error()
    assert call(y=rows(20, 33)) == -1 and "wide" in error()
    assert call(act=4) == -1 and "activation" in error()
    assert call(act=-1) == -1 and "activation" in error()
    assert call(bias=FAKE + 2) == -1 and "bias" in error()
    assert call(res=rows(19, 32)) == -1 and "residual" in error()
    assert call(res=rows(20, 31)) == -1 and "residual" in error()
    assert call(res=rows(20, 32, kind=1)) == -1 and "residual" in error()
    assert call(r=routing(11)) == -1 and "rows" in error()
    assert call(r=routing(experts=5)) == -1 and "experts" in error()
    assert call(r=routing(offsets=None)) == -1 and "null" in error()
    assert call(by_slot=1) == -1 and "slots" in error()
    assert call(r=None) == -1 and "routing" in error()
    assert call(r=None, w=weights(1), by_slot=1) == -1 and "routing" in error()
    assert call(r=None, w=weights(1)) == -1 and "20 rows" in error()
    assert call(y=rows(20, 32, stride=0)) == -1 and "stride" in error()
    assert call(kept=codes(19)) == -1 and call(kept=codes(width=33)) == -1 and call(kept=codes(data=FAKE + 4)) == -1
    assert call(kept=codes(scales=None)) == -1


def test_bias_gradient_refusals():
    lib = _lib.load()
    size = lib.ginex_bias_gradient_workspace_bytes
    assert size(-1, 4, 64) == 0 and size(10, 0, 64) == 0 and size(10, 1025, 64) == 0 and size(10, 4, 0) == 0
    assert size(0, 1, 1) > 0 and size(1 << 30, 1, 64) < 1 << 30
    big = 1 << 40
    assert lib.ginex_bias_gradient(ref(rows(19)), ref(routing()), FAKE, FAKE, big, None) == -1 and "slots" in error()
    assert lib.ginex_bias_gradient(ref(rows(20)), ref(routing()), None, FAKE, big, None) == -1
    assert lib.ginex_bias_gradient(ref(rows(20)), ref(routing()), FAKE, None, big, None) == -1
    assert lib.ginex_bias_gradient(ref(rows(20)), ref(routing()), FAKE, FAKE + 8, big, None) == -1
    assert lib.ginex_bias_gradient(ref(rows(20)), ref(routing()), FAKE, FAKE, 16, None) == -3 and "need" in error()


def test_expert_layer_refusals():
    lib = _lib.load()
    size = lib.ginex_expert_layer_workspace_bytes
    assert size(65, 2, 4, 64, 64) == 0 and "rows" in error()
    assert size(-1, 2, 4, 64, 64) == 0 and size(1, 0, 4, 64, 64) == 0 and size(1, 5, 4, 64, 64) == 0
    assert size(1, 17, 64, 64, 64) == 0 and size(1, 1, 1025, 64, 64) == 0 and size(0, 1, 1, 1, 1) > 0

    def call(x=rows(), router=rows(4), w=weights(), bias=None, top=2, act=0, y=rows(10, 32), ws=FAKE, n=1 << 40):
        return lib.ginex_expert_layer(ref(x), ref(router), ref(w), bias, top, act, ref(y), ws, n, None)

    assert call(router=rows(5)) == -1 and "experts" in error()
    assert call(router=rows(4, 63)) == -1 and "width" in error()
    assert call(router=rows(4, kind=1)) == -1 and "type" in error()
    assert call(w=weights(kind=1)) == -1 and "type" in error()
    assert call(w=weights(width=65)) == -1 and "wide" in error()
    assert call(y=rows(10, 33)) == -1 and "wide" in error()
    assert call(y=rows(9, 32)) == -1 and "rows" in error()
    assert call(x=rows(65), y=rows(65, 32)) == -1 and "rows" in error()
    assert call(top=5) == -1 and call(top=0) == -1 and call(act=9) == -1 and call(bias=FAKE + 3) == -1
    assert call(ws=None) == -1 and call(ws=FAKE + 4) == -1 and call(n=16) == -3 and "need" in error()


def test_layer_norm_refusals():
    lib, x = _lib.load(), rows()
    size = lib.ginex_layer_norm_backward_workspace_bytes
    assert size(-1, 8) == 0 and size(1 << 31, 8) == 0 and size(8, 0) == 0 and size(0, 1) > 0
    assert lib.ginex_layer_norm(ref(x), None, None, -1.0, ref(x), None, None) == -1 and "eps" in error()
    assert lib.ginex_layer_norm(ref(x), None, None, float("nan"), ref(x), None, None) == -1 and "eps" in error()
    assert lib.ginex_layer_norm(ref(x), FAKE + 2, None, 0.0, ref(x), None, None) == -1 and "weight" in error()
    assert lib.ginex_layer_norm(ref(x), None, FAKE + 2, 0.0, ref(x), None, None) == -1 and "bias" in error()
    assert lib.ginex_layer_norm(ref(x), None, None, 0.0, ref(x), FAKE + 4, None) == -1 and "stats" in error()
    assert lib.ginex_layer_norm(ref(x), None, None, 0.0, ref(rows(9)), None, None) == -1 and "rows" in error()
    assert lib.ginex_layer_norm(ref(x), None, None, 0.0, ref(rows(kind=1)), None, None) == -1 and "type" in error()

    def call(dy=x, stats=FAKE, w=None, dx=x, dw=FAKE, db=FAKE, ws=FAKE, n=1 << 40):
        return lib.ginex_layer_norm_backward(ref(dy), ref(x), stats, w, ref(dx), dw, db, ws, n, None)

    assert call(dy=rows(11)) == -1 and call(dx=rows(width=63)) == -1 and call(stats=None) == -1 and call(w=FAKE + 1) == -1
    assert call(dw=None) == -1 and "together" in error()
    assert call(db=FAKE + 2) == -1 and call(ws=None) == -1 and call(ws=FAKE + 128) == -1
    assert call(n=16) == -3 and "need" in error()


def test_lookup_refusals():
    lib, table, out = _lib.load(), rows(), rows(30)
    size = lib.ginex_lookup_backward_workspace_bytes
    assert size(-1, 8, 8) == 0 and size((1 << 30) + 1, 8, 8) == 0 and size(8, -1, 8) == 0 and size(8, 8, 0) == 0
    assert size(0, 0, 1) > 0
    assert lib.ginex_lookup(ref(table), None, 0, 1.0, ref(out), None) == -1 and "ids" in error()
    assert lib.ginex_lookup(ref(table), FAKE + 4, 1, 1.0, ref(out), None) == -1 and "ids" in error()
    assert lib.ginex_lookup(ref(table), FAKE, 2, 1.0, ref(out), None) == -1 and "ids_64" in error()
    assert lib.ginex_lookup(ref(table), FAKE, 0, 1.0, ref(rows(30, 63)), None) == -1 and "width" in error()
    assert lib.ginex_lookup(ref(table), FAKE, 0, 1.0, ref(rows(30, stride=0)), None) == -1 and "stride" in error()

    def call(dy=out, ids=FAKE, wide=0, dtable=table, ws=FAKE, n=1 << 40):
        return lib.ginex_lookup_backward(ref(dy), ids, wide, 1.0, ref(dtable), ws, n, None)

    assert call(ids=None) == -1 and call(wide=3) == -1 and call(dtable=rows(kind=1)) == -1 and call(ws=None) == -1
    assert call(ws=FAKE + 8) == -1 and call(n=16) == -3 and "need" in error()


def test_the_binding_refuses_tensors_elsewhere():
    import torch

    import paper_2208_09151_amd as g
    x, w = torch.zeros((3, 8)), torch.zeros((8, 4))
    for call in (lambda: g.linear(x, w), lambda: g.linear_backward(x, w), lambda: g.bias_gradient(x), lambda: g.layer_norm(x),
                 lambda: g.expert_layer(x, x, w[None], 1), lambda: g.lookup(x, torch.zeros(3, dtype=torch.int64)),
                 lambda: g.lookup_backward(x, torch.zeros(3, dtype=torch.int64), 4),
                 lambda: g.layer_norm_backward(x, x, torch.zeros((3, 2)))):
        with pytest.raises(ValueError, match="GPU memory"):
            call()
