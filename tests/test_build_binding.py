"""The library builds without what only the Python binding takes, and the binding is built anew for another Python or torch."""
import os
import subprocess

import pytest

from paper_2502_11880_b200 import build as b


@pytest.fixture
def elsewhere(monkeypatch, tmp_path):
    """Outputs go to a folder of their own; compilers are not run but recorded."""
    calls = []

    def run(cmd, check):
        calls.append(cmd)
        open(cmd[cmd.index("-o") + 1], "w").close()

    monkeypatch.setattr(b, "LIB", str(tmp_path / "lib.so"))
    monkeypatch.setattr(b, "BINDING", str(tmp_path / "binding.so"))
    monkeypatch.setattr(b, "OBJ_DIR", str(tmp_path / "build"))
    monkeypatch.setattr(subprocess, "run", run)
    return calls


def binding_calls(calls):
    return [c for c in calls if b.BINDING_SRC in c]


def test_library_without_a_cxx_compiler(monkeypatch, elsewhere):
    monkeypatch.setenv("CXX", "no-such-compiler")
    with pytest.warns(UserWarning, match="no-such-compiler"):
        assert b.build() == b.LIB
    assert os.path.exists(b.LIB) and not os.path.exists(b.BINDING) and not binding_calls(elsewhere)


def test_library_without_python_headers(monkeypatch, elsewhere, tmp_path):
    monkeypatch.setattr(b.sysconfig, "get_paths", lambda: {"include": str(tmp_path)})
    with pytest.warns(UserWarning, match="Python.h"):
        assert b.build() == b.LIB
    assert os.path.exists(b.LIB) and not binding_calls(elsewhere)


def test_binding_is_rebuilt_for_another_torch(monkeypatch, elsewhere):
    import torch
    b.build()
    b.build()
    assert len(binding_calls(elsewhere)) == 1                       # nothing has changed
    monkeypatch.setattr(torch, "__version__", "9.9.9")
    b.build()
    b.build()
    assert len(binding_calls(elsewhere)) == 2
    monkeypatch.setattr(b.sysconfig, "get_python_version", lambda: "9.9")
    b.build()
    assert len(binding_calls(elsewhere)) == 3


def test_a_compile_that_fails_raises(monkeypatch, elsewhere):
    def fails(cmd, check):
        if b.BINDING_SRC in cmd:
            raise subprocess.CalledProcessError(1, cmd)
        open(cmd[cmd.index("-o") + 1], "w").close()

    monkeypatch.setattr(subprocess, "run", fails)
    with pytest.raises(subprocess.CalledProcessError):
        b.build()
    assert os.path.exists(b.LIB)                                    # for those who do without the binding
