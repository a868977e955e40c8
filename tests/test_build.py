"""The build: the C library needs nothing of what _marshal.so needs, and _marshal.so is built for the torch and Python that load it."""
import os
import subprocess

import pytest
import torch

from paper_2412_00099_b200 import binding as mb
from paper_2412_00099_b200 import build as mbuild


@pytest.fixture
def elsewhere(tmp_path, monkeypatch):
    """_marshal.so and its stamp in an empty folder; commands are recorded and leave an empty file."""
    commands = []

    def run(cmd, **kw):
        commands.append(cmd)
        open(cmd[cmd.index("-o") + 1], "w").close()
        return subprocess.CompletedProcess(cmd, 0, "", "")
    monkeypatch.setattr(mbuild, "MARSHAL", str(tmp_path / "_marshal.so"))
    monkeypatch.setattr(mbuild, "OBJ", str(tmp_path / "obj"))
    monkeypatch.setattr(mbuild.subprocess, "run", run)
    return commands


@pytest.mark.parametrize("error", [RuntimeError("g++ failed"), FileNotFoundError("g++"), ModuleNotFoundError("torch")], ids=lambda e: type(e).__name__)
def test_the_library_is_built_without_the_marshalling(monkeypatch, capsys, error):
    mbuild.build()
    order = []

    def failing(force=False):
        order.append("marshal")
        raise error
    monkeypatch.setattr(mbuild, "build_marshal", failing)
    monkeypatch.setattr(mbuild, "_build_library", lambda *a: order.append("library"), raising=False)
    monkeypatch.setattr(mbuild, "_newest", lambda paths: float("inf"))         # everything is out of date
    assert mbuild.build() == mbuild.LIB
    assert order == ["library", "marshal"] and "_marshal.so was not built" in capsys.readouterr().err


def test_no_nvcc_on_the_path(elsewhere, monkeypatch, tmp_path):
    monkeypatch.setenv("NVCC", "no-such-compiler")
    home = tmp_path / "cuda"
    (home / "include").mkdir(parents=True)
    (home / "include" / "cuda_runtime_api.h").write_text("")
    monkeypatch.setenv("CUDA_HOME", str(home))
    mbuild.build_marshal()
    assert str(home / "include") in elsewhere[0]
    monkeypatch.setattr(mbuild.os.path, "exists", lambda p: False)
    with pytest.raises(RuntimeError, match="CUDA headers"):
        mbuild.build_marshal(force=True)


def test_built_again_for_another_torch(elsewhere, monkeypatch):
    mbuild.build_marshal()
    assert os.path.exists(mbuild.MARSHAL) and len(elsewhere) == 1
    mbuild.build_marshal()
    assert len(elsewhere) == 1
    monkeypatch.setattr(torch, "__version__", "0.0")
    mbuild.build_marshal()
    assert len(elsewhere) == 2 and any("torch 0.0" in a for a in elsewhere[1])
    mbuild.build_marshal()
    assert len(elsewhere) == 2


def test_the_binding_refuses_a_module_built_for_another_torch(monkeypatch):
    mbuild.build_marshal()
    monkeypatch.setattr(mb, "_fast", None)
    assert mb._marshal().built_for == mbuild.marshal_target()
    monkeypatch.setattr(mb, "_fast", None)
    monkeypatch.setattr(torch, "__version__", "0.0")
    with pytest.raises(mb.McceError, match="built for"):
        mb._marshal()
