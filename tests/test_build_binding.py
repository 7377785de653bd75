"""The solver's library is built whatever becomes of the losses' binding to torch; no compiler runs here."""
import os
import subprocess
import sys

import pytest

from paper_2203_16340_amd import build as B


@pytest.fixture
def runs(monkeypatch, tmp_path):
    """Commands that build() runs; every one with an output writes it."""
    seen = []

    def run(cmd, check):
        assert check
        seen.append(cmd)
        if cmd[0] == "g++" and run.gpp is not None:
            raise run.gpp
        with open(cmd[cmd.index("-o") + 1], "w") as f:
            f.write(" ".join(cmd))

    run.gpp = None
    monkeypatch.setattr(B.subprocess, "run", run)
    monkeypatch.setattr(B, "LIB", str(tmp_path / "liblbfgsb.so"))
    monkeypatch.setattr(B, "BINDING", str(tmp_path / "_losses.so"))
    with open(B.BINDING, "w") as f:
        f.write("of an older library")
    return run, seen


def test_both_are_built(runs):
    assert B.build() == B.LIB and os.path.exists(B.LIB)
    assert "older" not in open(B.BINDING).read()


def test_without_a_host_compiler(runs, capsys):
    runs[0].gpp = FileNotFoundError(2, "No such file or directory", "g++")
    assert B.build() == B.LIB and os.path.exists(B.LIB)
    assert not os.path.exists(B.BINDING) and "g++" in capsys.readouterr().err


def test_without_torch(runs, monkeypatch, capsys):
    monkeypatch.setitem(sys.modules, "torch", None)
    assert B.build() == B.LIB and os.path.exists(B.LIB)
    assert not os.path.exists(B.BINDING) and "torch" in capsys.readouterr().err


def test_a_binding_that_does_not_compile_is_an_error_after_the_library(runs):
    runs[0].gpp = subprocess.CalledProcessError(1, "g++")
    with pytest.raises(subprocess.CalledProcessError):
        B.build()
    assert os.path.exists(B.LIB) and not os.path.exists(B.BINDING)
