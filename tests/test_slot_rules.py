"""The rules of csrc/slots.hpp and tiling.hpp, compiled for the CPU: whatever offsets a routing holds, what the kernels
compute from them stays inside the arrays; which shape a weight gradient's sizes reach (no GPU)."""
import ctypes as C
import os
import random
import shutil
import subprocess

import pytest

import weight_shapes

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
i64 = C.c_int64
FOREIGN = [0, 1, 3, 4, 5, -1, -5, 1 << 31, 1 << 48, (1 << 48) + 1, 1 << 50, (1 << 63) - 1, -(1 << 63)]


@pytest.fixture(scope="module")
def rules(tmp_path_factory):
    if shutil.which("g++") is None:
        pytest.skip("no g++ here")
    lib = str(tmp_path_factory.mktemp("rules") / "rules.so")
    made = subprocess.run(["g++", "-O1", "-std=c++17", "-Wall", "-Werror", "-ftrapv", "-shared", "-fPIC",
                           "-I", os.path.join(ROOT, "paper_2208_09151_amd", "csrc"),
                           os.path.join(ROOT, "tests", "slot_rules.cpp"), "-o", lib], capture_output=True, text=True)
    assert made.returncode == 0, made.stderr
    lib = C.CDLL(lib)
    lib.rules_first_free_chunk.restype = i64
    lib.rules_first_free_chunk.argtypes = [i64, i64, C.c_uint32]
    lib.rules_ranges.restype = C.c_int32
    lib.rules_ranges.argtypes = [C.POINTER(i64), C.c_int32, i64, C.c_int32, C.c_int32]
    return lib


@pytest.mark.parametrize("chunks", [1, 2, 8192, 1 << 18])
@pytest.mark.parametrize("slots", [0, 4, (1 << 31) - 1])
@pytest.mark.parametrize("end", FOREIGN)
def test_rows_are_cleared_from_a_slot_on_that_exists(rules, end, slots, chunks):
    assert rules.rules_first_free_chunk(end, slots, chunks) == min(max(end, 0), slots) * chunks


def ranges(rules, offsets, slots, count, made_here):
    return rules.rules_ranges((i64 * len(offsets))(*offsets), len(offsets) - 1, slots, count, int(made_here))


def test_ranges_share_their_slots_out(rules):
    """Offsets as route() makes them: every slot once, and the parts that are added up are those that were left."""
    rng = random.Random(1)
    for _ in range(3000):
        experts, count = rng.choice([1, 2, 8, 63, 64, 65, 200]), rng.choice([1, 2, 3, 7, 8, 32, 128, 512])
        most = rng.choice([0, 1, 20, 300, 5000, 10 ** 6])
        offsets = [0]
        for _ in range(experts):
            offsets.append(offsets[-1] + (0 if rng.random() < 0.3 else rng.randrange(most + 1)))
        slots = offsets[-1] + rng.choice([0, 1, 1000])
        assert ranges(rules, offsets, slots, count, True) == 0, (offsets, slots, count)
    assert ranges(rules, [0, (1 << 31) - 1], (1 << 31) - 1, 512, True) == 0


def test_ranges_of_offsets_made_elsewhere(rules):
    """Offsets that descend, or that no slot has: no slot and no part that is not there."""
    assert ranges(rules, [0, 1000, 2000, 16], 2048, 16, False) == 0
    rng = random.Random(2)
    for _ in range(20_000):
        experts, count = rng.choice([1, 2, 3, 8, 65, 130]), rng.choice([1, 2, 3, 16, 64, 512])
        slots = rng.choice([0, 1, 16, 100, 2048, 10 ** 6, (1 << 31) - 1])
        offsets = [rng.choice(FOREIGN) if rng.random() < 0.2 else rng.randrange(slots + 1) for _ in range(experts + 1)]
        if rng.random() < 0.5:
            offsets[:-1] = sorted(offsets[:-1])
        assert ranges(rules, offsets, slots, count, False) == 0, (offsets, slots, count)


def tiling(rules, dtype, slots, experts, width, out):
    found = (C.c_int32 * 6)()
    rules.rules_tiling(1 if dtype == "bf16" else 2, i64(slots), experts, i64(width), i64(out), found)
    return tuple(found)


@pytest.mark.parametrize("shape, sizes, width, out, dtype", weight_shapes.PARAMS, ids=weight_shapes.IDS)
def test_sizes_reach_the_shape_that_they_are_there_for(rules, shape, sizes, width, out, dtype):
    found = tiling(rules, dtype, sum(sizes) + weight_shapes.EMPTY, len(sizes), width, out)
    assert found[:4] == shape


def test_every_shape_has_sizes_of_every_type(rules):
    shapes = set()
    for dtype in weight_shapes.TYPES:
        for slots in (1, 1000, 50_000, 300_000, 2_000_000):
            for width in (5, 40, 100, 200, 700):
                for out in (5, 20, 40, 100, 200, 700):
                    shapes.add((tiling(rules, dtype, slots, 8, width, out)[:4], dtype))
    assert shapes == {(shape, dtype) for shape, _, _, _, dtype in weight_shapes.PARAMS}
