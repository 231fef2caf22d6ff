"""build.py's decisions, with a stand-in for the compilers: the library does not depend on the optional module _marshal."""
import subprocess

import pytest
import torch

from paper_2506_07366_b200 import binding, build


@pytest.fixture
def compilers(monkeypatch, tmp_path):
    """Paths of a fresh tree and compilers that write an empty result, or fail where `broken` names them."""
    monkeypatch.setattr(build, "LIB_PATH", str(tmp_path / "lib.so"))
    monkeypatch.setattr(build, "MARSHAL_PATH", str(tmp_path / "_marshal.so"))

    class Compilers:
        broken, ran = set(), []

    def run(cmd, **_):
        name = cmd[0].rsplit("/", 1)[-1]
        Compilers.ran.append(name)
        if name in Compilers.broken:
            return subprocess.CompletedProcess(cmd, 1, "", f"{name}: no such header")
        if name + " missing" in Compilers.broken:
            raise FileNotFoundError(name)
        open(cmd[cmd.index("-o") + 1], "wb").close()
        return subprocess.CompletedProcess(cmd, 0, "", "")

    Compilers.ran = []
    monkeypatch.setattr(build.subprocess, "run", run)
    return Compilers


@pytest.mark.parametrize("broken", ["g++", "g++ missing"])
def test_library_is_built_without_a_host_compiler(compilers, capsys, tmp_path, broken):
    compilers.broken = {broken}
    (tmp_path / "_marshal.so").write_bytes(b"of an older source")
    assert build.build(force=True) == build.LIB_PATH
    assert (tmp_path / "lib.so").exists() and compilers.ran == ["nvcc", "g++"]
    assert "_marshal" in capsys.readouterr().err
    assert not (tmp_path / "_marshal.so").exists()        # what could not be renewed is not used


def test_both_are_built(compilers, tmp_path):
    build.build()
    assert (tmp_path / "lib.so").exists() and (tmp_path / "_marshal.so").exists()


def test_library_failure_is_an_error(compilers):
    compilers.broken = {"nvcc"}
    with pytest.raises(RuntimeError, match="nvcc"):
        build.build(force=True)


def test_marshal_of_another_torch_is_not_used_and_is_rebuilt(compilers, monkeypatch):
    """It reads torch's C++ objects, whose layout belongs to one version."""
    build.build()
    open(build.MARSHAL_PATH, "wb").write(b"..." + build.marshal_marker().encode() + b"...")
    compilers.ran.clear()
    build.build()
    assert compilers.ran == []                            # both are current
    monkeypatch.setattr(torch, "__version__", "0.0.1")
    build.build()
    assert compilers.ran == ["g++"]


def test_binding_ignores_a_marshal_of_another_torch(monkeypatch):
    build.build_marshal()
    assert binding._marshal() is not None
    monkeypatch.setattr(torch, "__version__", "0.0.1")
    assert binding._marshal() is None
