"""include/ginex_train.h: every entry point is exported and bound, and refuses what it cannot do before
anything is launched (no GPU)."""
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


def codes(n=10, width=64, data=FAKE, scales=FAKE):
    return _lib.CodesDesc(n, width, data, scales)


def ref(x):
    return None if x is None else C.byref(x)


def test_every_declared_symbol_is_exported_and_bound():
    text = open(os.path.join(ROOT, "include", "ginex_train.h")).read()
    text = re.sub(r"/\*.*?\*/", "", text, flags=re.S)
    names = sorted(set(re.findall(r"\b(ginex_[a-z_]+)\s*\(", text)))
    assert sorted(_lib.TRAIN_SIGNATURES) == names and len(names) == 10
    for n in names:
        assert getattr(_lib.load(), n) is not None


def test_constants_of_the_binding_are_the_headers():
    from paper_2208_09151_amd import training
    text = open(os.path.join(ROOT, "include", "ginex_train.h")).read()
    value = {k: int(v) for k, v in re.findall(r"#define GINEX_(\w+) (\d+)", text)}
    assert training.CODE_BLOCK == value["CODE_BLOCK"]
    assert training.ACTIVATIONS == {"relu": value["ACT_RELU"], "silu": value["ACT_SILU"], "gelu": value["ACT_GELU"]}
    assert sorted(training._TYPES.values()) == [value["F32"], value["BF16"], value["F16"]]


@pytest.mark.parametrize("args, says", [
    ((-1, 2, 4), "rows=-1"), ((10, 0, 4), "top=0"), ((10, 65, 4), "top=65"), ((10, 2, 0), "experts=0"),
    ((10, 2, 1025), "experts=1025"), ((1 << 30, 2, 4), "pairs"), ((1 << 40, 1, 4), "pairs")])
def test_route_sizes(args, says):
    assert _lib.load().ginex_route_workspace_bytes(*args) == 0
    assert says in error()


def test_route_refusals():
    lib = _lib.load()

    def call(out=routing(), chosen=FAKE, wide=1, ws=FAKE, ws_bytes=1 << 30):
        return lib.ginex_route(chosen, wide, -1, ref(out), ws, ws_bytes, None)

    assert call(out=None) == -1 and "null" in error()
    assert call(chosen=None) == -1
    assert call(chosen=FAKE + 4) == -1 and "misaligned" in error()
    assert call(out=routing(offsets=None)) == -1
    assert call(out=routing(slot=None)) == -1
    assert call(out=routing(source=FAKE + 2)) == -1
    assert call(ws=None) == -1
    assert call(ws=FAKE + 8) == -1
    assert call(out=routing(n=100_000), ws_bytes=16) == -3 and "need" in error()
    assert lib.ginex_route_workspace_bytes(100_000, 2, 64) > lib.ginex_route_workspace_bytes(10, 2, 64) > 0


BAD_ROWS = [(rows(kind=3), "type"), (rows(width=0), "width"), (rows(width=(1 << 20) + 1), "width"),
            (rows(stride=63), "stride"), (rows(data=None), "null"), (rows(data=FAKE + 2), "aligned"),
            (rows(n=-1), "rows")]


@pytest.mark.parametrize("bad, says", BAD_ROWS)
def test_rows_that_no_call_takes(bad, says):
    lib, good, slots, kept = _lib.load(), rows(), rows(20), codes()
    r = routing()
    assert lib.ginex_dispatch(ref(r), ref(bad), ref(slots), None) == -1 and says in error()
    assert lib.ginex_dispatch(ref(r), ref(good), ref(bad), None) == -1
    assert lib.ginex_combine(ref(r), ref(bad), FAKE, ref(good), None) == -1 and says in error()
    assert lib.ginex_combine_backward(ref(r), ref(bad), ref(slots), FAKE, ref(slots), FAKE, None) == -1
    assert lib.ginex_compress(ref(bad), 0, None, ref(kept), None) == -1 and says in error()
    assert lib.ginex_restore(ref(kept), ref(bad), None) == -1 and says in error()
    assert lib.ginex_activate_backward(ref(kept), 1, ref(bad), ref(good), None) == -1 and says in error()
    assert lib.ginex_weight_gradient(ref(kept), ref(r), ref(bad), FAKE, FAKE, 1 << 40, None) == -1 and says in error()


def test_rows_that_do_not_fit_each_other():
    lib, r = _lib.load(), routing()
    assert lib.ginex_dispatch(ref(r), ref(rows(11)), ref(rows(20)), None) == -1 and "11" in error()
    assert lib.ginex_dispatch(ref(r), ref(rows(10)), ref(rows(21)), None) == -1 and "slots" in error()
    assert lib.ginex_dispatch(ref(r), ref(rows(10)), ref(rows(20, kind=1)), None) == -1 and "type" in error()
    assert lib.ginex_dispatch(ref(r), ref(rows(10)), ref(rows(20, width=65)), None) == -1 and "width" in error()
    assert lib.ginex_dispatch(ref(r), ref(rows(10)), ref(rows(20, stride=0)), None) == -1 and "stride" in error()
    assert lib.ginex_dispatch(None, ref(rows(10)), ref(rows(20)), None) == -1
    assert lib.ginex_combine(ref(r), ref(rows(19)), FAKE, ref(rows(10)), None) == -1
    assert lib.ginex_combine(ref(r), ref(rows(20)), FAKE + 2, ref(rows(10)), None) == -1
    assert lib.ginex_combine_backward(ref(r), ref(rows(10)), ref(rows(20)), None, ref(rows(20)), FAKE, None) == -1
    assert lib.ginex_combine_backward(ref(r), ref(rows(10)), ref(rows(20)), FAKE, ref(rows(20)), None, None) == -1


def test_codes_refusals():
    lib, x = _lib.load(), rows()
    assert lib.ginex_compress(ref(x), 0, None, None, None) == -1
    assert lib.ginex_compress(ref(x), 0, None, ref(codes(data=None)), None) == -1
    assert lib.ginex_compress(ref(x), 0, None, ref(codes(data=FAKE + 4)), None) == -1 and "aligned" in error()
    assert lib.ginex_compress(ref(x), 0, None, ref(codes(9)), None) == -1 and "codes" in error()
    assert lib.ginex_compress(ref(x), 0, None, ref(codes(width=65)), None) == -1
    assert lib.ginex_compress(ref(x), 4, ref(x), ref(codes()), None) == -1 and "activation" in error()
    assert lib.ginex_compress(ref(x), 1, None, ref(codes()), None) == -1
    assert lib.ginex_compress(ref(x), 0, ref(x), ref(codes()), None) == -1
    assert lib.ginex_compress(ref(x), 1, ref(rows(kind=1)), ref(codes()), None) == -1
    assert lib.ginex_activate_backward(ref(codes()), 0, ref(x), ref(x), None) == -1 and "activation" in error()
    assert lib.ginex_activate_backward(ref(codes()), 2, ref(x), ref(rows(9)), None) == -1
    assert lib.ginex_restore(ref(codes(8)), ref(x), None) == -1


def test_weight_gradient_refusals():
    lib = _lib.load()
    size = lib.ginex_weight_gradient_workspace_bytes
    assert size(-1, 4, 64, 64) == 0 and "slots" in error()
    assert size(10, 0, 64, 64) == 0 and size(10, 4, 0, 64) == 0 and size(10, 4, 64, 0) == 0
    assert size(10, 1025, 64, 64) == 0 and size(0, 4, 64, 64) > 0
    assert size(10, 4, 1 << 17, 1 << 16) == 0 and "too many" in error()

    def call(kept=codes(), r=routing(), dy=rows(20), dw=FAKE, ws=FAKE, ws_bytes=1 << 40):
        return lib.ginex_weight_gradient(ref(kept), ref(r), ref(dy), dw, ws, ws_bytes, None)

    assert call(kept=None) == -1
    assert call(r=routing(n=11)) == -1 and "routing" in error()
    assert call(dy=rows(10)) == -1 and "slots" in error()
    assert call(r=None) == -1                       # 20 rows of dy for 10 rows
    assert call(dw=None) == -1
    assert call(ws=None) == -1
    assert call(ws=FAKE + 128) == -1
    big = dict(kept=codes(1_000_000), r=routing(1_000_000), dy=rows(2_000_000))
    assert call(**big, ws_bytes=16) == -3 and "need" in error()


def test_the_binding_refuses_tensors_elsewhere():
    import torch

    import paper_2208_09151_amd as g
    with pytest.raises(ValueError, match="GPU memory"):
        g.route(torch.zeros((3, 2), dtype=torch.int64), 4)
    with pytest.raises(ValueError, match="GPU memory"):
        g.compress(torch.zeros((3, 64)))
    with pytest.raises(ValueError, match="GPU memory"):
        g.Compressed(torch.zeros((3, 64), dtype=torch.int8), torch.zeros((3, 2), dtype=torch.uint8), 64)
    with pytest.raises(ValueError, match="activation"):
        g.activate(torch.zeros((3, 64)), "tanh")
