"""The compiled torch front end is optional: a build without g++, torch or its headers leaves the library and says so, a
module made for another torch is built again and not used until then."""
import os
import sys

import pytest

from paper_1906_04585_b200 import build as B


@pytest.fixture
def apart(tmp_path, monkeypatch):
    """The front end's files in a folder of their own, and a library that needs no work."""
    monkeypatch.setattr(B, "FRONT_LIB", str(tmp_path / "_front.so"))
    monkeypatch.setattr(B, "FRONT_STAMP", str(tmp_path / "made" / "front.torch"))
    monkeypatch.setattr(B, "_stale", lambda: False)
    return tmp_path


def compiles(monkeypatch, times):
    def command(out):
        times.append(out)
        return ["touch", out]
    monkeypatch.setattr(B, "_front_command", command)


@pytest.mark.parametrize("command", [["false"], ["no-such-compiler"]])
def test_a_compiler_that_fails_is_reported(apart, monkeypatch, capsys, command):
    monkeypatch.setattr(B, "_front_command", lambda out: command)
    assert B.build() == B.LIB
    said = capsys.readouterr().err
    assert "_front.so is not built" in said and "Python" in said
    assert not os.path.exists(B.FRONT_LIB)


def test_without_torch(apart, monkeypatch, capsys):
    monkeypatch.setitem(sys.modules, "torch", None)
    assert B.build() == B.LIB
    assert "ModuleNotFoundError" in capsys.readouterr().err and not os.path.exists(B.FRONT_LIB)


def test_a_failed_build_takes_the_old_one_away(apart, monkeypatch, capsys):
    times = []
    compiles(monkeypatch, times)
    B.build()
    monkeypatch.setattr(B, "_torch_version", lambda: "another")
    monkeypatch.setattr(B, "_front_command", lambda out: ["false"])
    B.build()
    assert not os.path.exists(B.FRONT_LIB)


def test_built_once_for_a_torch_and_its_sources(apart, monkeypatch):
    times = []
    compiles(monkeypatch, times)
    B.build()
    B.build()
    assert len(times) == 1 and os.path.exists(B.FRONT_LIB)
    monkeypatch.setattr(B, "_torch_version", lambda: "another")
    B.build()
    B.build()
    assert len(times) == 2
    os.utime(B.FRONT_LIB, (1, 1))       # older than front.cpp
    B.build()
    assert len(times) == 3


def test_a_missing_front_end_does_not_build_the_library_again(tmp_path, monkeypatch):
    B.build()
    monkeypatch.setattr(B, "FRONT_LIB", str(tmp_path / "_front.so"))
    assert B._front_stale() and not B._stale()


def test_the_module_of_another_torch_is_not_used(monkeypatch):
    torch = pytest.importorskip("torch")
    B.build()
    from paper_1906_04585_b200 import sequence as S
    if S._front is None:
        pytest.skip("no compiled front end here")
    assert S._front.torch_version == torch.__version__
    with pytest.warns(UserWarning, match="torch 0.1"):
        monkeypatch.setattr(S._front, "torch_version", "0.1")
        assert S._compiled() is None
