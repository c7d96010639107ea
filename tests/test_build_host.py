"""The library for C callers is built whatever becomes of the Python module that needs torch's headers (no compiler is run here)."""
import os

import pytest

from paper_2406_06484_amd import build_ext


@pytest.fixture
def stand_ins(monkeypatch, tmp_path):
    """compiling leaves empty objects, linking writes its output"""
    done = []

    def link(cmd):
        done.append("link")
        open(cmd[cmd.index("-o") + 1], "w").close()

    monkeypatch.setattr(build_ext, "OUT", str(tmp_path / "lib.so"))
    monkeypatch.setattr(build_ext, "BINDING", str(tmp_path / "_attention.so"))
    monkeypatch.setattr(build_ext, "_compile", lambda src: str(tmp_path / src))
    monkeypatch.setattr(build_ext.subprocess, "check_call", link)
    return done


def test_a_failing_module_is_reported_behind_the_library(stand_ins, monkeypatch):
    def broken():
        raise RuntimeError("g++ failed")

    monkeypatch.setattr(build_ext, "_compile_binding", broken)
    with pytest.raises(RuntimeError, match=r"g\+\+ failed"):
        build_ext.build(verbose=False)
    assert stand_ins == ["link"] and os.path.exists(build_ext.OUT)


@pytest.mark.parametrize("missing", ["torch", "g++"])
def test_without_torch_or_a_host_compiler_there_is_a_library_and_a_word_about_the_module(stand_ins, monkeypatch, capfd, missing):
    if missing == "torch":
        monkeypatch.setitem(__import__("sys").modules, "torch", None)
    else:
        def no_compiler(*a, **kw):
            raise FileNotFoundError(2, "No such file or directory", "g++")
        monkeypatch.setattr(build_ext.subprocess, "run", no_compiler)
    assert build_ext.build(verbose=False) == build_ext.OUT
    assert stand_ins == ["link"] and os.path.exists(build_ext.OUT) and not os.path.exists(build_ext.BINDING)
    assert "_attention.so" in capfd.readouterr().err and missing in missing
