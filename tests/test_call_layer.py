"""CPU: the native call layer is built behind the library, for one torch and Python, and loaded by the calls that take it."""
import os
import shutil
import subprocess

import pytest

import paper_2607_24555_b200 as locks
from paper_2607_24555_b200 import binding, build


@pytest.fixture
def in_tree():
    return build.build_calls()


@pytest.fixture
def other_path(tmp_path, monkeypatch):
    path = str(tmp_path / "_calls.so")
    monkeypatch.setattr(binding, "_CALLS_PATH", path)
    monkeypatch.setattr(binding, "_calls_module", None)
    return path


def test_a_module_of_another_torch_is_not_loaded(other_path):
    with pytest.raises(locks.LocksError, match="missing"):
        binding.calls()
    build.build_calls()
    data = open(other_path, "rb").read()
    assert data.count(binding.calls_stamp().encode()) == 1 and not build.calls_stale()
    with open(other_path, "wb") as f:   # never loaded, so that it need not be whole
        f.write(data.replace(b"torch " + binding.torch.__version__.encode(), b"torch 0" + binding.torch.__version__.encode()[1:]))
    assert build.calls_stale()
    with pytest.raises(locks.LocksError, match="another torch"):
        binding.calls()


def test_the_library_builds_where_the_call_layer_cannot(other_path, monkeypatch, capsys):
    ran = []

    class Done:
        returncode, stdout, stderr = 0, "", ""
    monkeypatch.setattr(subprocess, "run", lambda cmd, **kw: ran.append(cmd[0]) or Done())
    monkeypatch.setattr(build.shutil, "which", lambda name: None)
    open(other_path, "w").write("stale")
    assert build.build(force=True) == build.LIB and not os.path.exists(other_path)
    assert [os.path.basename(c) for c in ran] == ["nvcc"] and "_calls.so is not built" in capsys.readouterr().err
    # with a compiler: behind the library, and a failure of it says so
    monkeypatch.setattr(build.shutil, "which", lambda name: "/usr/bin/" + name)
    build.build(force=True)
    assert [os.path.basename(c) for c in ran] == ["nvcc", "nvcc", "g++"]

    class Failed(Done):
        returncode, stderr = 1, "no such header"
    monkeypatch.setattr(subprocess, "run", lambda cmd, **kw: Failed() if cmd[0] == "g++" else Done())
    with pytest.raises(RuntimeError, match="no such header"):
        build.build(force=True)


class _Context(locks.Context):
    """A context whose library handle is made up: calls of the native layer are refused before they use it."""

    def __init__(self, handle):
        self.cfg, self.k, self.summary_bytes = binding.make_config(4, 2, 8, "i4", "bf16", 2, 4, 32), 2, 832
        self.device, self.handle = binding.torch.device("cuda", 0), handle

    def close(self):
        self.handle = None


def test_contexts_take_the_call_layer_when_a_call_does(in_tree, other_path):
    """Contexts are made, closed and used by the other calls without it."""
    ctx = _Context(binding.C.c_void_p(1))
    assert "_calls" not in ctx.__dict__
    with pytest.raises(locks.LocksError, match="missing"):
        ctx.locks_rope(None, None, None, None)
    with pytest.raises(AttributeError):
        ctx.no_such_call
    shutil.copy(in_tree, other_path)
    with pytest.raises(locks.LocksError, match="needed"):
        ctx.locks_rope(None, None, None, None)
    closed = _Context(None)
    with pytest.raises(locks.LocksError, match="closed"):
        closed.locks_rope(None, None, None, None)
