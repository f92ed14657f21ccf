"""The reader of PyTorch's tensors belongs to the PyTorch and the Python that it was built for."""
import os
import subprocess
import sys

import pytest
import torch

from paper_1910_11141_amd import build
from paper_1910_11141_amd import learning as G


def test_what_it_was_built_for():
    assert build.torch_version() == torch.__version__
    assert build.reader_fits()


@pytest.mark.parametrize("change", [("torch_version", lambda: "0.1.2+none"), ("PYTHON", "cpython-99")])
def test_another_pytorch_or_python(change, monkeypatch):
    """It is not loaded, and built again."""
    monkeypatch.setattr(build, *change)
    monkeypatch.setattr(G, "_tensors", None)
    with pytest.raises(ImportError, match="another PyTorch or Python"):
        G.nuts_norm([torch.zeros(3)])
    assert G._tensors is None
    run = []
    monkeypatch.setattr(build, "is_stale", lambda: False)
    monkeypatch.setattr(build, "sources", lambda: [])
    monkeypatch.setattr(build.subprocess, "run", lambda cmd, check: run.append(os.path.basename(cmd[cmd.index("-o") + 1])))
    assert build.build(force=False) == build.LIB_PATH and "libnuts_tensors.so" in run


def test_a_reader_that_says_nothing(monkeypatch, tmp_path):
    (tmp_path / "old.so").write_bytes(b"\x7fELF" + bytes(100))
    for path, word in ((tmp_path / "old.so", "another PyTorch or Python"), (tmp_path / "none.so", "missing")):
        monkeypatch.setattr(build, "TENSORS_LIB", str(path))
        monkeypatch.setattr(G, "TENSORS_PATH", str(path))
        monkeypatch.setattr(G, "_tensors", None)
        with pytest.raises(ImportError, match=word):
            G.nuts_norm([torch.zeros(3)])


def test_the_package_needs_no_pytorch_for_its_version():
    subprocess.run([sys.executable, "-c", "import sys; from paper_1910_11141_amd import build; build.torch_version(), build.reader_fits(); assert 'torch' not in sys.modules"],
                   check=True)
