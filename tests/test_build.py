"""What the build does where something is missing or out of date; compilers are replaced by ones that only take notes."""
import os
import sys

import pytest

from paper_2506_07533_b200 import build as B


@pytest.fixture
def compilers(monkeypatch, tmp_path):
    """Commands in the order in which they are started; every output file is written (empty) somewhere else."""
    started = []

    class Compiler:
        returncode = 0

        def __init__(self, cmd, **_):
            started.append(cmd)
            out = cmd[cmd.index("-o") + 1]
            assert str(out).startswith(str(tmp_path))
            with open(out, "wb") as f:
                f.write(" ".join(cmd).encode())

        def communicate(self):
            return "", None

    monkeypatch.setattr(B.subprocess, "Popen", Compiler)
    monkeypatch.setattr(B.subprocess, "check_call", Compiler)
    monkeypatch.setattr(B, "HERE", str(tmp_path))
    monkeypatch.setattr(B, "LIB", str(tmp_path / "libmoqae.so"))
    monkeypatch.setattr(B, "MARSHAL", str(tmp_path / "_marshal.so"))
    return started


def is_library(cmd):
    return "nvcc" in os.path.basename(cmd[0])


def test_the_library_comes_first(compilers):
    assert B.build() == B.LIB and os.path.exists(B.LIB) and os.path.exists(B.MARSHAL)
    assert [is_library(c) for c in compilers] == [True] * (len(B.SOURCES) + 1) + [False]
    del compilers[:]
    B.build()                                                # nothing has changed
    assert not compilers


@pytest.mark.parametrize("lacks", ["torch", "headers"])
def test_the_library_needs_no_torch(compilers, monkeypatch, tmp_path, lacks, capsys):
    """A machine with nvcc alone builds the C library, as it always has."""
    if lacks == "torch":
        monkeypatch.setitem(sys.modules, "torch", None)
    else:
        import torch
        monkeypatch.setattr(torch, "__file__", str(tmp_path / "torch" / "__init__.py"))
    assert B.build() == B.LIB and os.path.exists(B.LIB) and not os.path.exists(B.MARSHAL)
    assert compilers and all(is_library(c) for c in compilers)
    assert "_marshal.so is left out" in capsys.readouterr().err


def test_the_module_is_built_again_for_another_torch(compilers, monkeypatch):
    """It holds layouts of torch's objects, so its age alone does not say that it fits."""
    import torch
    B.build_marshal()
    B.build_marshal()
    assert len(compilers) == 1
    monkeypatch.setattr(torch, "__version__", "9.9.9")
    B.build_marshal()
    B.build_marshal()
    assert len(compilers) == 2


def test_a_module_for_another_torch_is_refused(monkeypatch):
    from paper_2506_07533_b200 import binding as mq
    B.build()
    monkeypatch.setattr(mq, "_MARSHAL", None)
    assert mq._native().built_for == B.marshal_key()
    monkeypatch.setattr(mq, "_MARSHAL", None)
    monkeypatch.setattr(B, "marshal_key", lambda: "torch 9.9.9")
    with pytest.raises(RuntimeError, match="built for another torch"):
        mq._native()
    assert mq._MARSHAL is None
