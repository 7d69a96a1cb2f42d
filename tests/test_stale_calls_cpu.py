"""A relation_calls.so that is stale, broken or left from a failed build is not used: the serving calls
then run through Python, with a warning.  CPU only."""
import os
import shutil
import subprocess
from types import SimpleNamespace

import pytest
import torch

from paper_2608_20172_gb300 import binding
from paper_2608_20172_gb300 import build as libbuild


@pytest.fixture(scope="module")
def built():
    libbuild.build()
    if libbuild.build_calls() is None:
        pytest.skip("the native calls cannot be built here")
    return libbuild.CALLS


@pytest.fixture
def copy(built, monkeypatch, tmp_path):
    """The built file and its stamp in a place of their own, not loaded yet."""
    path = str(tmp_path / "relation_calls.so")
    shutil.copy(built, path)
    shutil.copy(built + ".stamp", path + ".stamp")
    monkeypatch.setattr(binding, "CALLS_PATH", path)
    monkeypatch.setattr(binding, "_calls", None)
    monkeypatch.setattr(libbuild, "BUILD", str(tmp_path))
    monkeypatch.setattr(libbuild, "CALLS", path)
    return path


def test_current(copy, recwarn):
    assert binding._native() is not binding._NoCalls and not recwarn.list


def test_absent(copy, recwarn):
    os.remove(copy)
    assert binding._native() is binding._NoCalls and not recwarn.list


def test_broken(copy):
    with open(copy, "wb") as f:
        f.write(b"not a library")
    with pytest.warns(RuntimeWarning, match="relation_calls"):
        assert binding._native() is binding._NoCalls
    assert binding._native() is binding._NoCalls  # (asked once)


@pytest.mark.parametrize("stamp", ["other sources", None])
def test_of_other_sources(copy, stamp):
    os.remove(copy + ".stamp")
    if stamp:
        with open(copy + ".stamp", "w") as f:
            f.write(stamp)
    with pytest.warns(RuntimeWarning, match="relation_calls"):
        assert binding._native() is binding._NoCalls


def test_for_another_torch(copy, monkeypatch):
    monkeypatch.setattr(torch, "__version__", "0.0")
    with pytest.warns(RuntimeWarning, match="relation_calls"):
        assert binding._native() is binding._NoCalls


def test_another_cuda_path_is_the_same_file(copy, monkeypatch, recwarn):
    monkeypatch.setenv("CUDA_HOME", "/somewhere/else")
    assert binding._native() is not binding._NoCalls and not recwarn.list


@pytest.mark.parametrize("how", ["compiler fails", "no compiler"])
def test_a_failed_build_leaves_nothing_old(copy, monkeypatch, how, capsys):
    def run(cmd, **_):
        if how == "no compiler":
            raise FileNotFoundError("g++")
        return SimpleNamespace(returncode=1, stderr="no such header", stdout="")
    monkeypatch.setattr(subprocess, "run", run)
    assert libbuild.build_calls(force=True) is None
    assert "not built" in capsys.readouterr().err
    assert not os.path.exists(copy) and not os.path.exists(copy + ".stamp")
    assert binding._native() is binding._NoCalls
