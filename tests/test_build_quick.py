"""The layers' compiled calls are a part that the library does without (no GPU): where they cannot be built, build() tells and
goes on, and nothing half made is left."""
import os
import subprocess

import pytest

from paper_2208_09151_amd import build as b


@pytest.fixture
def place(tmp_path, monkeypatch):
    pytest.importorskip("torch")
    monkeypatch.setattr(b, "QUICK", str(tmp_path / "_quick.so"))
    return tmp_path


def write(command, text):
    with open(command[command.index("-o") + 1], "w") as f:
        f.write(text)


def test_a_whole_one_takes_its_place(place, monkeypatch):
    (place / "_quick.so").write_text("an older one")
    monkeypatch.setattr(subprocess, "check_call", lambda command: write(command, "whole"))
    b._build_quick()
    assert os.listdir(place) == ["_quick.so"] and (place / "_quick.so").read_text() == "whole"


@pytest.mark.parametrize("there", [False, True])
@pytest.mark.parametrize("error", [FileNotFoundError("g++"), PermissionError("g++"), subprocess.CalledProcessError(1, "g++")])
def test_no_compiler_or_none_that_gets_through(place, monkeypatch, error, there):
    def fail(command):
        write(command, "half of one")
        raise error

    if there:
        (place / "_quick.so").write_text("an older one")
    monkeypatch.setattr(subprocess, "check_call", fail)
    with pytest.warns(UserWarning, match="not built"):
        b._build_quick()
    assert os.listdir(place) == []


@pytest.mark.parametrize("name, value", [("__version__", "2.10.1+rocm7.0"), ("__version__", "2.10"), ("git_version", "0" * 40)])
def test_one_for_another_torch_is_not_loaded(monkeypatch, name, value):
    """Whatever the times of the files say: compiled calls use torch's classes as they were described to them."""
    import torch

    from paper_2208_09151_amd import _lib
    if _lib.quick() is None:
        pytest.skip("the compiled calls are not built")
    monkeypatch.setattr(torch if name == "__version__" else torch.version, name, value)
    assert _lib.quick() is None
