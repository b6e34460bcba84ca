"""What a build needs: the CUDA library needs nvcc alone, the marshalling module of `spec` a C++ compiler and torch (CPU)."""
import os
import shutil
import subprocess

import pytest

from paper_2511_21862_b200 import binding, build


@pytest.fixture(scope="module", autouse=True)
def _built():
    build.build()


@pytest.fixture
def calls(tmp_path, monkeypatch):
    """A copy of the marshalling module, as the one that builds look at."""
    path = str(tmp_path / "_spec_calls.so")
    shutil.copy(build.CALLS, path)
    monkeypatch.setattr(build, "CALLS", path)
    return path


@pytest.mark.parametrize("how", ["no compiler", "compiler fails", "no torch"])
def test_the_cuda_library_is_built_without_the_marshalling_module(calls, monkeypatch, capsys, how):
    real = subprocess.run

    def run(cmd, **kw):
        if cmd[0] != "g++":
            return real(cmd, **kw)
        if how == "no compiler":
            raise FileNotFoundError(2, "No such file or directory", "g++")
        return subprocess.CompletedProcess(cmd, 1, "", "Python.h: No such file or directory")

    monkeypatch.setattr(subprocess, "run", run)
    if how == "no torch":
        def no_torch():
            raise ModuleNotFoundError("No module named 'torch'")
        monkeypatch.setattr(build, "_built_for", no_torch)
    else:
        monkeypatch.setattr(build, "_built_for", lambda: "torch of another day")
    assert build.build() == build.LIB and os.path.exists(build.LIB)
    assert not os.path.exists(calls)                    # one that may not fit is not left to be loaded
    assert "_spec_calls.so could not be built" in capsys.readouterr().err
    assert binding.lib().ooco_version() > 0
    with pytest.raises((RuntimeError, OSError, ImportError)):
        build.build_calls()


def test_the_marshalling_module_is_rebuilt_for_another_torch(calls, monkeypatch):
    assert not build.is_stale(calls)
    monkeypatch.setattr(build, "_built_for", lambda: "torch 1.0 python 3.1")
    assert build.is_stale(calls)


def test_a_module_of_another_torch_is_not_used(monkeypatch):
    from paper_2511_21862_b200 import spec
    spec._lib()
    monkeypatch.setattr(spec, "_L", None)
    monkeypatch.setattr(spec, "_calls", None)
    monkeypatch.setattr(build, "_built_for", lambda: "torch 1.0 python 3.1")
    with pytest.raises(ImportError, match="paper_2511_21862_b200.build"):
        spec._lib()
