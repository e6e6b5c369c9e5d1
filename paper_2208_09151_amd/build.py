"""Builds libginex.so (gfx950 HIP kernels + C ABI) in-tree with hipcc.

hipcc cross-compiles for gfx950 without a GPU, so this runs anywhere the ROCm toolchain is
installed.  ``python -m paper_2208_09151_amd.build`` or ``build()``.
"""
from __future__ import annotations

import os
import subprocess
import sys
import warnings
from concurrent.futures import ThreadPoolExecutor

PKG = os.path.dirname(os.path.abspath(__file__))
ROOT = os.path.dirname(PKG)
CSRC = os.path.join(PKG, "csrc")
OBJ = os.path.join(PKG, "_build")
LIB = os.path.join(PKG, "libginex.so")
QUICK = os.path.join(PKG, "_quick.so")
SOURCES = ["core.cpp", "gather.hip", "sampler.hip", "changeset.hip", "neighbor_cache.hip",
           "static_policy.hip", "route.hip", "rows.hip", "codes.hip", "weights.hip", "linear.hip", "resident.hip", "few.hip",
           "bias.hip", "norm.hip", "lookup.hip"]
HIPCC = os.environ.get("HIPCC", "/opt/rocm/bin/hipcc")
FLAGS = ["-O3", "--offload-arch=gfx950", "-fPIC", "-std=c++17", "-Wall",
         "-Xclang", "-target-feature", "-Xclang", "-packed-fp32-ops",
         "-I", os.path.join(ROOT, "include"), "-I", CSRC]


def _compile(src: str) -> str:
    obj = os.path.join(OBJ, os.path.splitext(src)[0] + ".o")
    cmd = [HIPCC, *FLAGS, "-x", "hip", "-c", os.path.join(CSRC, src), "-o", obj]
    r = subprocess.run(cmd, capture_output=True, text=True)
    # the host pass does not know the packed-fp32 feature switch and says so: harmless
    err = "\n".join(l for l in r.stderr.splitlines() if "packed-fp32-ops" not in l)
    if r.returncode != 0:
        raise RuntimeError(f"hipcc failed on {src}:\n{err}")
    if err.strip():
        sys.stderr.write(err + "\n")
    return obj


def _build_quick() -> None:
    """The layers' calls without the interpreter's part (csrc/quick.cpp), against the installed torch.  Without it the Python
    names do the same, so that a compiler that is missing or does not get through is told and is no error."""
    try:
        import sysconfig

        import torch
        from torch.utils import cpp_extension

        from ._lib import quick_is_for
    except ImportError:
        return
    lib = os.path.join(os.path.dirname(torch.__file__), "lib")
    include = [*cpp_extension.include_paths(), sysconfig.get_paths()["include"], os.path.join(ROOT, "include")]
    made = f"{QUICK[:-3]}.{os.getpid()}.so"         # (in its place once it is whole)
    command = ["g++", "-O2", "-std=c++17", "-Wall", "-fPIC", "-shared", "-D__HIP_PLATFORM_AMD__", "-DUSE_ROCM",
               f"-D_GLIBCXX_USE_CXX11_ABI={int(torch._C._GLIBCXX_USE_CXX11_ABI)}", f'-DGINEX_QUICK_IS_FOR="{quick_is_for()}"',
               *(f"-isystem{p}" for p in include),
               os.path.join(CSRC, "quick.cpp"), "-o", made, "-L", lib, "-ltorch", "-ltorch_cpu", "-lc10", "-ltorch_python",
               "-L", PKG, "-lginex", "-Wl,-rpath,$ORIGIN"]
    try:
        subprocess.check_call(command)
        os.replace(made, QUICK)
    except (OSError, subprocess.CalledProcessError) as e:
        warnings.warn(f"the layers' compiled calls are not built, their Python names do without: {e}")
        for half_or_old in (made, QUICK):
            if os.path.exists(half_or_old):
                os.remove(half_or_old)


def build(verbose: bool = False) -> str:
    os.makedirs(OBJ, exist_ok=True)
    with ThreadPoolExecutor(max_workers=4) as ex:
        objs = list(ex.map(_compile, SOURCES))
    cmd = [HIPCC, "--offload-arch=gfx950", "-shared", "-fPIC", *objs, "-o", LIB]
    subprocess.check_call(cmd)
    _build_quick()
    if verbose:
        print("built", LIB)
    return LIB


if __name__ == "__main__":
    build(verbose=True)
