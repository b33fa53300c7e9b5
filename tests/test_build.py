"""The build without a GPU: the library does not need what the compiled way in for torch tensors needs."""
import os
import subprocess

import pytest

from paper_2602_00608_b200 import build


@pytest.mark.parametrize("how", ["no g++", "g++ fails"])
def test_the_library_is_built_where_the_torch_module_cannot_be(monkeypatch, tmp_path, capsys, how):
    """A module of an earlier build does not stay beside a library whose descriptors may be others."""
    old = tmp_path / "_vd_torch.so"
    old.write_bytes(b"an earlier build's")
    os.utime(old, (1, 1))
    monkeypatch.setattr(build, "TORCH_LIB", str(old))
    run = subprocess.run

    def without(cmd, *a, **kw):
        if cmd[0] != "g++":
            return run(cmd, *a, **kw)
        if how == "no g++":
            raise FileNotFoundError("g++")
        return subprocess.CompletedProcess(cmd, 1, "", "error: no such header")

    monkeypatch.setattr(subprocess, "run", without)
    assert build.build() == build.LIB and os.path.exists(build.LIB)
    assert not old.exists()
    assert "_vd_torch.so was not built" in capsys.readouterr().err


def test_the_torch_module_is_built_here():
    build.build()
    assert os.path.exists(build.TORCH_LIB)
