"""When the compiled part of the binding is made again, and what happens where it cannot be made."""
import os
import subprocess
import sysconfig

import pytest
import torch

import paper_2605_26845_b200 as ms
from paper_2605_26845_b200 import build as cuda_build


@pytest.fixture
def compiled(monkeypatch, tmp_path):
    """Compilers that run nothing: they write their command, as a compiler does its strings, to the output. Returns the commands."""
    commands = []

    def run(command, check):
        assert check
        commands.append(command)
        with open(command[command.index("-o") + 1], "wb") as f:
            f.write("\0".join(c.replace('="', "\0").rstrip('"') for c in command).encode() + b"\0")

    monkeypatch.setattr(subprocess, "run", run)
    monkeypatch.setattr(cuda_build, "BINDING", str(tmp_path / "_binding.so"))
    for name in ("LIB", "LIB_CHECKED"):
        monkeypatch.setattr(cuda_build, name, str(tmp_path / f"{name}.so"))
    monkeypatch.setattr(cuda_build, "HERE", str(tmp_path / "package"))
    monkeypatch.setattr(cuda_build.os.path, "getmtime", lambda p, real=os.path.getmtime: real(p) if os.path.exists(p) else 0.0)
    return commands


def made(commands):
    n = len(commands)
    commands.clear()
    return n


def test_the_binding_goes_with_one_torch_one_python_and_one_set_of_flags(compiled, monkeypatch):
    cuda_build.build_binding()
    assert made(compiled) == 1
    cuda_build.build_binding()
    assert made(compiled) == 0
    for name, value in (("__version__", "9.9.9"), ("compiled_with_cxx11_abi", lambda: not torch._C._GLIBCXX_USE_CXX11_ABI)):
        with monkeypatch.context() as m:
            m.setattr(torch, name, value)
            cuda_build.build_binding()
            assert made(compiled) == 1, name
            cuda_build.build_binding()
            assert made(compiled) == 0, name
        cuda_build.build_binding()
        assert made(compiled) == 1, name
    with monkeypatch.context() as m:
        m.setattr(sysconfig, "get_config_var", lambda name, real=sysconfig.get_config_var: "cpython-399" if name == "SOABI" else real(name))
        cuda_build.build_binding()
        assert made(compiled) == 1
    with monkeypatch.context() as m:
        m.setenv("CXX", "another-g++")
        cuda_build.build_binding()
        assert made(compiled) == 1
    cuda_build.build_binding(force=True)
    assert made(compiled) == 1
    os.utime(cuda_build.BINDING, (0, 0))                     # older than its source
    cuda_build.build_binding()
    assert made(compiled) == 1


def test_the_library_is_built_where_the_binding_cannot_be(compiled, monkeypatch):
    def fails(force=False):
        raise subprocess.CalledProcessError(1, "g++")

    monkeypatch.setattr(cuda_build, "build_binding", fails)
    for checked, lib in ((False, cuda_build.LIB), (True, cuda_build.LIB_CHECKED)):
        with pytest.raises(subprocess.CalledProcessError):   # (which is said)
            cuda_build.build(checked=checked)
        assert os.path.exists(lib) and made(compiled) == len(cuda_build.SOURCES) + 1


def test_a_binding_of_another_torch_is_not_loaded(monkeypatch):
    cuda_build.build()
    monkeypatch.setattr(ms, "_bound", None)
    x, w = torch.zeros((4, 8)), torch.zeros(8)
    with monkeypatch.context() as m:
        m.setattr(torch, "__version__", "9.9.9")
        with pytest.raises(ms.MoeschedError, match="another torch.*build"):
            ms.rms_norm(x, w)
        m.setattr(cuda_build, "BINDING", "/nowhere/_binding.so")
        with pytest.raises(ms.MoeschedError, match="nowhere.*build"):
            ms.rms_norm(x, w)
    with pytest.raises(ms.MoeschedError, match="must be a CUDA tensor"):
        ms.rms_norm(x, w)
    assert ms._bound.stamp.startswith(cuda_build.made_for()) and cuda_build.holds(cuda_build.BINDING, ms._bound.stamp)
