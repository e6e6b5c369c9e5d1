"""What the meeting of k_few_experts' workgroups rests on, in the instructions that the compiler makes of it (no GPU): answers are
stored and loaded past the dies' caches, and no pair is counted before the stores in front of it have arrived."""
import os
import re
import subprocess

import pytest

from paper_2208_09151_amd import build as b


@pytest.fixture(scope="module")
def kernels(tmp_path_factory):
    if not os.path.exists(b.HIPCC):
        pytest.skip("hipcc is not installed")
    to = str(tmp_path_factory.mktemp("listing") / "few.s")
    subprocess.run([b.HIPCC, *b.FLAGS, "-x", "hip", "--cuda-device-only", "-S", os.path.join(b.CSRC, "few.hip"), "-o", to], check=True,
                   capture_output=True)
    found = re.findall(r"\n(\w*k_few_experts\w*):.*?\n(.*?)\.Lfunc_end", open(to).read(), re.S)
    return {name: [line.split(";")[0].split() for line in body.splitlines() if re.match(r"\t[a-z]", line)] for name, body in found}


def test_stores_counts_and_loads(kernels):
    assert len(kernels) == 18                       # three types, two orders of weights, three numbers of waves
    for name, lines in kernels.items():
        count, = [i for i, line in enumerate(lines) if line[0].startswith("global_atomic_add")]
        stores = [i for i, line in enumerate(lines[:count]) if line[0].startswith("global_store")]
        assert stores and all("sc1" in lines[i] for i in stores), name
        between = [" ".join(line) for line in lines[stores[-1]:count]]
        waits = [i for i, line in enumerate(between) if line.startswith("s_waitcnt vmcnt(0)")]
        barriers = [i for i, line in enumerate(between) if line == "s_barrier"]
        assert waits and barriers and waits[0] < barriers[0], name
        behind = lines[count:]
        assert [line[0] for line in behind].index("s_barrier") < min(i for i, line in enumerate(behind) if "sc1" in line), name
        assert sum("sc1" in line and line[0].startswith("global_load") for line in behind) == 16, name         # answers in flight
