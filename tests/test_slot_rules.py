"""The rules of csrc/slots.hpp, compiled for the CPU: whatever offsets a routing holds, what the kernels compute from
them stays inside the arrays (no GPU)."""
import ctypes as C
import os
import shutil
import subprocess

import pytest

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
    return lib


@pytest.mark.parametrize("chunks", [1, 2, 8192, 1 << 18])
@pytest.mark.parametrize("slots", [0, 4, (1 << 31) - 1])
@pytest.mark.parametrize("end", FOREIGN)
def test_rows_are_cleared_from_a_slot_on_that_exists(rules, end, slots, chunks):
    assert rules.rules_first_free_chunk(end, slots, chunks) == min(max(end, 0), slots) * chunks
