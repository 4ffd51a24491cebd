"""The build without a part of what it can use: no compiler is run."""

import importlib.util
import os
import types

import pytest

from paper_2004_09362_gb300 import build


@pytest.fixture
def box(tmp_path, monkeypatch):
    """Places and commands of a build that only makes empty files; `failing` is what a command that fails has in it."""
    b = types.SimpleNamespace(ran=[], failing=None, torch=tmp_path / "torch", out=tmp_path / "libgar.so", marshal=tmp_path / "_marshal.so")
    b.torch.mkdir()
    (b.torch / "version.py").write_text("__version__ = '1'")
    monkeypatch.setattr(build, "OUT", str(b.out))
    monkeypatch.setattr(build, "MARSHAL", str(b.marshal))
    monkeypatch.setattr(build, "BUILD", str(tmp_path / "build"))
    monkeypatch.setattr(build, "_nvcc", lambda: "/nowhere/bin/nvcc")

    def run(cmd, **kw):
        line = " ".join(cmd)
        if b.failing == "missing" and cmd[0] == "g++":
            raise FileNotFoundError(cmd[0])
        failed = b.failing is not None and b.failing in line
        if not failed:
            b.ran.append(line)
            open(cmd[cmd.index("-o") + 1], "w").close()
        return types.SimpleNamespace(returncode=int(failed), stdout="", stderr="")

    monkeypatch.setattr(build.subprocess, "run", run)
    spec = types.SimpleNamespace(submodule_search_locations=[str(b.torch)])
    b.spec = spec
    monkeypatch.setattr(importlib.util, "find_spec", lambda name: b.spec if name == "torch" else None)
    return b


def test_without_torch_the_library_is_built(box):
    box.spec = None
    assert build.build() == str(box.out)
    assert box.out.exists() and not box.marshal.exists()
    n = len(box.ran)
    build.build()                           # and not built again
    assert len(box.ran) == n


@pytest.mark.parametrize("failing", ["marshal.cpp", "_marshal.so", "missing"])
def test_a_binding_that_fails_leaves_the_library_built(box, failing):
    box.failing = failing
    with pytest.raises(RuntimeError, match="marshal"):
        build.build()
    assert box.out.exists() and not box.marshal.exists()
    box.failing, n = None, len(box.ran)
    build.build()                           # what failed, and only that
    assert box.marshal.exists() and all("marshal" in line for line in box.ran[n:])


def test_another_torch_has_the_binding_built_again(box):
    build.build()
    n = len(box.ran)
    build.build()
    assert len(box.ran) == n
    (box.torch / "version.py").write_text("__version__ = '2'")
    build.build()
    assert len(box.ran) == n + 2 and all("marshal" in line for line in box.ran[n:])
    os.remove(box.out)
    build.build()
    assert box.out.exists() and len(box.ran) == n + 2 + len(build.SOURCES) + 1
