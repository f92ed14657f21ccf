"""The library is built where PyTorch, or what the reader of its tensors is compiled with, is missing (paper_1910_11141_amd/build.py)."""
import importlib.util
import os
import re
import subprocess

import pytest

from paper_1910_11141_amd import build


@pytest.fixture
def commands(monkeypatch):
    """Nothing is compiled; what would be is listed."""
    run = []

    def pretend(cmd, check):
        run.append(cmd)
        if "-c" in cmd:
            open(re.sub(r"\.hip\.o$", "-hip-amdgcn-amd-amdhsa-gfx950.s", cmd[-1]), "w").close()

    monkeypatch.setattr(build.subprocess, "run", pretend)
    return run


def names(commands):
    return [os.path.basename(cmd[cmd.index("-o") + 1]) for cmd in commands]


def test_all_of_it(commands):
    assert build.build() == build.LIB_PATH
    assert {"libnuts_hip.so", "libnuts_ubench.so", "libnuts_tensors.so", "nuts_step.hip.o"} <= set(names(commands)) and len(commands) == len(build.sources()) + 3


@pytest.mark.parametrize("force", [True, False])
def test_without_pytorch(commands, monkeypatch, force):
    find = importlib.util.find_spec
    monkeypatch.setattr(importlib.util, "find_spec", lambda name, *more: None if name == "torch" else find(name, *more))
    monkeypatch.setattr(build, "is_stale", lambda: True)
    assert build.build(force=force, verbose=True) == build.LIB_PATH
    assert names(commands)[-1] == "libnuts_hip.so" and "libnuts_ubench.so" in names(commands) and "libnuts_tensors.so" not in names(commands)


def test_nothing_is_built_again_for_want_of_pytorch(commands, monkeypatch, tmp_path):
    find = importlib.util.find_spec
    monkeypatch.setattr(importlib.util, "find_spec", lambda name, *more: None if name == "torch" else find(name, *more))
    made = tmp_path / "libnuts_ubench.so"
    made.touch()
    monkeypatch.setattr(build, "is_stale", lambda: False)
    monkeypatch.setattr(build, "UBENCH_LIB", str(made))
    monkeypatch.setattr(build, "TENSORS_LIB", str(tmp_path / "none"))
    assert build.build(force=False) == build.LIB_PATH and commands == []


@pytest.mark.parametrize("error", [FileNotFoundError("g++"), subprocess.CalledProcessError(1, "g++")])
def test_without_what_the_reader_is_compiled_with(commands, monkeypatch, error):
    """It is said, when the library is there."""
    pretend = build.subprocess.run

    def fails(cmd, check):
        if build.TENSORS_SRC in cmd:
            raise error
        pretend(cmd, check)

    monkeypatch.setattr(build.subprocess, "run", fails)
    with pytest.raises(type(error)):
        build.build()
    assert names(commands)[-1] == "libnuts_hip.so"
