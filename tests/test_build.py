"""What the build does where something is missing or fails, with stand-ins for the compilers, on the CPU: the C-ABI library needs hipcc alone."""
import os
import sys

import pytest

import __graft_entry__
import paper_2507_07966_amd as pa
from oracle import build as oracle_build
from paper_2507_07966_amd import build as b


@pytest.fixture
def place(tmp_path, monkeypatch):
    """A tree of its own for what is built, and compilers that write their output file and log their name; FAIL names a source that is not accepted."""
    for name in ("hipcc", "cxx"):
        with open(tmp_path / name, "w") as f:
            f.write('#!/bin/sh\nout=\nfor a in "$@"; do\n  case "$a" in *"${FAIL:-no source}") echo "$a is refused"; exit 1;; esac\n'
                    f'  [ "$prev" = "-o" ] && out=$a\n  prev=$a\ndone\necho {name} "$(basename "$out")" >> "$LOG"\necho {name} > "$out"\n')
        os.chmod(tmp_path / name, 0o755)
    monkeypatch.setenv("HIPCC", str(tmp_path / "hipcc"))
    monkeypatch.setenv("CXX", str(tmp_path / "cxx"))
    monkeypatch.setenv("LOG", str(tmp_path / "log"))
    monkeypatch.setattr(b, "HERE", str(tmp_path))
    monkeypatch.setattr(b, "LIB", str(tmp_path / "libprefix_attn.so"))
    monkeypatch.setattr(b, "BINDING", str(tmp_path / "_sampling.so"))
    return tmp_path


def built(place):
    return [(place / n).exists() for n in ("libprefix_attn.so", "_sampling.so")]


def test_library_and_module(place):
    assert b.build(out=b.LIB) == b.LIB and built(place) == [True, True]
    log = (place / "log").read_text().split("\n")
    assert log.index("hipcc libprefix_attn.so") < log.index("cxx _sampling.so")


def test_library_without_torch(place, monkeypatch, capfd):
    (place / "_sampling.so").write_text("of an earlier build")
    monkeypatch.setitem(sys.modules, "torch", None)   # importing it raises ImportError
    b.build(out=b.LIB)
    assert built(place) == [True, False] and "alone" in capfd.readouterr().err


def test_library_where_the_module_fails(place, monkeypatch, capfd):
    monkeypatch.setenv("FAIL", "py_sampling.cpp")
    with pytest.raises(RuntimeError, match="py_sampling.cpp"):
        b.build(out=b.LIB)
    assert built(place) == [True, False] and "is refused" in capfd.readouterr().err
    monkeypatch.setenv("CXX", str(place / "no such compiler"))
    with pytest.raises(RuntimeError, match="no such compiler"):
        b.build(out=b.LIB)
    assert built(place) == [True, False]


def test_a_failing_library_is_named(place, monkeypatch, capfd):
    monkeypatch.setenv("FAIL", "rope.hip")
    with pytest.raises(RuntimeError, match="hipcc"):
        b.build(out=b.LIB)
    assert built(place) == [False, False] and "rope.hip FAILED" in capfd.readouterr().err


def test_the_build_imports_what_it_built(monkeypatch):
    for module, name in ((b, "build"), (b, "build_probe"), (oracle_build, "build")):
        monkeypatch.setattr(module, name, lambda *a, **k: None)
    monkeypatch.setattr(pa.sampling, "_native", None)
    __graft_entry__.build()
    assert pa.sampling._native is not None
