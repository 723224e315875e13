"""What the in-tree build makes and when it makes it again, with a compiler that
only writes the files it is asked for."""
import os
import sys
import types

import pytest


@pytest.fixture
def build(monkeypatch, tmp_path):
    from paper_2504_18583_gb300 import _build as b
    for name in ("LIB", "BINDING", "BUILD", "BINDING_TORCH"):
        at = str(tmp_path / name.lower()) if name == "BUILD" else str(tmp_path / "build" / name.lower())
        monkeypatch.setattr(b, name, at, raising=False)
    os.makedirs(b.BUILD)
    b.commands, b.fail = [], ""

    def run(cmd, **kw):
        b.commands.append(cmd)
        if b.fail and any(b.fail in x for x in cmd):
            return types.SimpleNamespace(returncode=1, stdout="", stderr="made to fail")
        open(cmd[cmd.index("-o") + 1], "w").close()
        return types.SimpleNamespace(returncode=0, stdout="", stderr="")

    monkeypatch.setattr(b.subprocess, "run", run)
    yield b
    del b.commands, b.fail


def compiled(b, name):
    return sum(any(x.endswith(name) for x in c) for c in b.commands)


def test_the_library_needs_no_torch(build, monkeypatch):
    monkeypatch.setitem(sys.modules, "torch", None)  # as if it were not installed
    assert build.build() == build.LIB and os.path.exists(build.LIB)
    assert compiled(build, "torch_binding.cpp") == 0 and not os.path.exists(build.BINDING)
    assert build.up_to_date()
    monkeypatch.undo()


def test_another_torch_needs_another_binding(build, monkeypatch):
    import importlib.metadata
    build.build()
    assert compiled(build, "torch_binding.cpp") == 1 and os.path.exists(build.BINDING)
    assert build.up_to_date()
    build.build()
    assert compiled(build, "torch_binding.cpp") == 1
    monkeypatch.setattr(importlib.metadata, "version", lambda name: "0.0.1")
    assert not build.up_to_date()
    build.build()
    assert compiled(build, "torch_binding.cpp") == 2 and build.up_to_date()


def test_a_binding_that_fails_leaves_the_library(build):
    build.fail = "torch_binding.cpp"
    with pytest.raises(RuntimeError, match="torch_binding.cpp"):
        build.build()
    assert os.path.exists(build.LIB) and not build.up_to_date()
    build.fail = ""
    build.build()
    assert build.up_to_date()
