"""The bindings' compiled part needs a host compiler, Python's headers and PyTorch's (CPU).
The library needs none of them: without one its build goes on, and the bindings that need
the part raise.  What is there but does not compile fails the build."""
import shutil
import sys

import pytest

from paper_2504_03651_amd import build


@pytest.fixture
def stale(tmp_path, monkeypatch):
    """A part that an earlier build left, in place of the tree's own."""
    at = tmp_path / "_binding.so"
    at.write_bytes(b"of an earlier build")
    monkeypatch.setattr(build, "BINDING", str(at))
    return at


def _no_compiler(monkeypatch):
    monkeypatch.setenv("CXX", "no-such-compiler")


def _no_torch(monkeypatch):
    monkeypatch.setitem(sys.modules, "torch", None)


def _no_python_headers(monkeypatch):
    import sysconfig
    monkeypatch.setattr(sysconfig, "get_paths", lambda: {"include": "/no/such/folder"})


def _no_torch_headers(monkeypatch):
    import torch
    monkeypatch.setattr(torch, "__file__", "/no/such/folder/torch/__init__.py")


@pytest.mark.parametrize("take_away, what", [(_no_compiler, "no-such-compiler"), (_no_torch, "PyTorch"),
                                             (_no_python_headers, "Python.h"), (_no_torch_headers, "PyTorch's headers")])
def test_without_what_the_part_needs_the_library_is_built(stale, monkeypatch, capsys, take_away, what):
    take_away(monkeypatch)
    assert build.build_binding() is None
    assert not stale.exists(), "one that was built against another library may not stay"
    err = capsys.readouterr().err
    assert what in err and "int8.py, rope.py and norm.py" in err


@pytest.mark.skipif(shutil.which("g++") is None, reason="needs g++")
def test_what_does_not_compile_fails(stale, tmp_path, monkeypatch):
    (tmp_path / "binding.cpp").write_text("not C++")
    monkeypatch.setattr(build, "CSRC", str(tmp_path))
    with pytest.raises(RuntimeError, match="binding.cpp"):
        build.build_binding()
