"""How the library is built, without compiling anything."""
import sys

import pytest

from paper_2007_12216_amd import build


def commands_of_a_build(monkeypatch):
    run = []
    monkeypatch.setattr(build, "run_all", lambda commands, verbose: run.extend(commands) or "")
    assert build.build_library() == build.LIB
    return [c[0] for c in run], run


def test_the_library_needs_no_torch(monkeypatch):
    """The C library is compiled and linked where torch is absent; only decoder.py, which needs torch itself, calls the extension module."""
    monkeypatch.setitem(sys.modules, "torch", None)  # its import fails
    compilers, run = commands_of_a_build(monkeypatch)
    assert compilers == ["hipcc"] * 4 and build.LIB in run[-1]


def test_the_extension_module_comes_behind_the_library(monkeypatch):
    compilers, run = commands_of_a_build(monkeypatch)
    assert compilers == ["hipcc"] * 4 + ["g++"] and build.LIB in run[-2] and build.EXTENSION in run[-1]


def test_an_error_names_the_compiler_that_failed():
    """(the commands are this interpreter, in the compilers' place)"""
    fails, works = ([sys.executable, "-c", f"print({said!r}); raise SystemExit({code})"] for said, code in (("no such thing", 3), ("fine", 0)))
    with pytest.raises(RuntimeError) as e:
        build.run_all([works, fails], False)
    assert str(e.value).startswith(sys.executable + " failed:") and "no such thing" in str(e.value) and "hipcc" not in str(e.value)
    assert build.run_all([works, works], False).split() == ["fine", "fine"]
