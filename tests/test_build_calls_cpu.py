"""Building relation_calls.so is beside the library's build: where it cannot be built, build_calls returns
None and the library is built all the same."""
import sys

import pytest

from paper_2608_20172_gb300 import build as libbuild


@pytest.fixture
def place(monkeypatch, tmp_path):
    monkeypatch.setattr(libbuild, "BUILD", str(tmp_path))
    monkeypatch.setattr(libbuild, "CALLS", str(tmp_path / "relation_calls.so"))
    return tmp_path


def test_without_torch(place, monkeypatch, capsys):
    monkeypatch.setitem(sys.modules, "torch", None)  # (import raises ImportError)
    monkeypatch.setattr(libbuild, "_build_lib", lambda *a: "the library")
    assert libbuild.build_calls() is None
    assert "not built" in capsys.readouterr().err
    assert libbuild.build() == "the library"
