"""The build step with a compiler that only writes empty files: what it makes, in which order, and what stops it."""
import sys
import types

import pytest

from paper_2510_25977_amd import build as bld


@pytest.fixture
def compiler(monkeypatch, tmp_path):
    """Build into a folder of its own.  The fixture's value: the names of the files compiled or linked, and what fails."""
    state = types.SimpleNamespace(made=[], fails=set())

    def run(cmd, **kw):
        inputs = [c.rsplit("/", 1)[-1] for c in cmd if c.endswith((".hip", ".cpp"))]
        target = cmd[cmd.index("-o") + 1]
        if state.fails & set(inputs):
            return types.SimpleNamespace(returncode=1, stdout="", stderr="no")
        open(target, "w").close()
        state.made.append(target.rsplit("/", 1)[-1])
        return types.SimpleNamespace(returncode=0, stdout="", stderr="")

    monkeypatch.setattr(bld, "subprocess", types.SimpleNamespace(run=run))
    monkeypatch.setattr(bld, "OBJDIR", tmp_path / "_build")
    monkeypatch.setattr(bld, "LIB", tmp_path / "libsvdmlp.so")
    monkeypatch.setattr(bld, "TENSORS", tmp_path / "_tensors.so")
    return state


def test_a_build_makes_the_library_and_the_tensor_checks(compiler):
    assert bld.build(force=True) == bld.LIB
    assert bld.LIB.exists() and bld.TENSORS.exists()
    compiler.made.clear()
    assert bld.build(force=False) == bld.LIB and not compiler.made           # current
    bld.TENSORS.unlink()
    assert bld.build(force=False) == bld.LIB and bld.TENSORS.exists()


def test_the_library_needs_no_torch(compiler, monkeypatch, capsys):
    """The C boundary is built with hipcc alone; without torch there is no binding to build the tensor checks for."""
    monkeypatch.setitem(sys.modules, "torch", None)
    assert bld.build(force=True) == bld.LIB
    assert bld.LIB.exists() and not bld.TENSORS.exists()
    assert "_tensors.so" in capsys.readouterr().err
    compiler.made.clear()
    assert bld.build(force=False) == bld.LIB and not compiler.made


def test_the_library_is_there_when_the_host_compiler_fails(compiler):
    """... and the build says so, since the binding's operators need the rest."""
    compiler.fails = {"tensors.cpp"}
    with pytest.raises(RuntimeError, match="tensors.cpp"):
        bld.build(force=True)
    assert bld.LIB.exists() and not bld.TENSORS.exists()


def test_a_source_that_does_not_compile_stops_the_build(compiler):
    compiler.fails = {"norm.hip"}
    with pytest.raises(RuntimeError, match="norm.hip"):
        bld.build(force=True)
    assert not bld.LIB.exists()


def test_the_tensor_checks_are_rebuilt_for_another_torch(compiler, monkeypatch):
    """They are compiled against one torch and one Python: under another one they are not current, however new."""
    import torch
    bld.build(force=True)
    compiler.made.clear()
    bld.build(force=False)
    assert not compiler.made
    monkeypatch.setattr(torch, "__version__", "0.0.0")
    bld.build(force=False)
    assert "_tensors.so" in compiler.made
    compiler.made.clear()
    bld.build(force=False)
    assert not compiler.made
