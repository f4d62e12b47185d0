"""What the build makes of a machine without the tools for the C++ module (CPU; nothing is compiled)."""
import os
import sys
import sysconfig

import pytest

import paper_2203_00854_amd as P
from paper_2203_00854_amd import binding as B
from paper_2203_00854_amd import build as M


@pytest.fixture
def place(monkeypatch, tmp_path):
    """The build with its results in a folder of their own, a compiler for the GPU that always succeeds, and no other program on the path."""
    monkeypatch.setattr(M, "OBJ", str(tmp_path / "obj"))
    monkeypatch.setattr(M, "LIB", str(tmp_path / "libff.so"))
    monkeypatch.setattr(M, "CALLS", str(tmp_path / os.path.basename(M.CALLS)))
    monkeypatch.setattr(M, "HIPCC", "/bin/true")
    monkeypatch.setenv("PATH", str(tmp_path))
    return tmp_path


def program(place, text):
    path = place / "g++"
    path.write_text("#!/bin/sh\n" + text + "\n")
    path.chmod(0o755)


def test_the_module_is_this_interpreters():
    assert os.path.basename(M.CALLS) == "_calls" + sysconfig.get_config_var("EXT_SUFFIX")
    assert B.CALLS_PATH == M.CALLS and P.calls().__file__ == M.CALLS


def test_the_library_is_built_without_a_host_compiler(place, capsys):
    open(M.CALLS, "w").close()                                   # of an earlier build
    assert M.build() == M.LIB
    assert "g++" in capsys.readouterr().out and not os.path.exists(M.CALLS)


def test_the_library_is_built_without_torch(place, capsys, monkeypatch):
    program(place, "exit 0")
    monkeypatch.setitem(sys.modules, "torch", None)
    assert M.build() == M.LIB
    assert "torch" in capsys.readouterr().out


def test_the_library_is_built_without_the_interpreters_headers(place, capsys, monkeypatch):
    program(place, "exit 0")
    monkeypatch.setattr(M.sysconfig, "get_paths", lambda: {"include": str(place)})
    assert M.build() == M.LIB
    assert "Python.h" in capsys.readouterr().out


def test_a_failing_compilation_is_an_error(place):
    program(place, "echo no such thing >&2; exit 1")
    with pytest.raises(RuntimeError, match="no such thing"):
        M.build()


def test_a_missing_module_is_named(monkeypatch):
    monkeypatch.setattr(B, "_calls", None)
    monkeypatch.setattr(B, "CALLS_PATH", B.CALLS_PATH + ".none")
    with pytest.raises(FileNotFoundError, match="_calls"):
        P.calls()
