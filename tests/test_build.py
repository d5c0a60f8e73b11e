"""The library is built for C callers whatever becomes of the Python binding's module, and the module follows the PyTorch
it is compiled against.  (A small stand-in for the sources: these tests are about what is built when.)"""
import os

import pytest


@pytest.fixture
def tree(tmp_path, monkeypatch):
    from paper_2601_08670_gb300 import build
    src = tmp_path / "csrc"
    src.mkdir()
    (src / "one.cu").write_text('extern "C" int pced_one() { return 1; }\n')
    (src / "calls.cpp").write_text('extern "C" int pced_one();\nextern "C" int two() { return 1 + pced_one(); }\n')
    monkeypatch.setattr(build, "CSRC", str(src))
    monkeypatch.setattr(build, "LIBDIR", str(tmp_path / "lib"))
    monkeypatch.setattr(build, "LIB", str(tmp_path / "lib" / "libpced.so"))
    monkeypatch.setattr(build, "SOURCES", ["one.cu"])
    return build


def times(build):
    return [os.stat(f).st_mtime_ns for f in (build.LIB, os.path.join(build.LIBDIR, build.CALLS))]


def test_a_module_that_does_not_compile_costs_no_library(tree):
    with open(os.path.join(tree.CSRC, "calls.cpp"), "w") as f:
        f.write("#error no such header\n")
    with pytest.raises(RuntimeError, match="calls.cpp"):
        tree.build()
    assert os.path.exists(tree.LIB)


def test_a_module_out_of_date_is_not_left(tree):
    tree.build()
    with open(os.path.join(tree.CSRC, "calls.cpp"), "w") as f:
        f.write("#error no such header\n")
    later = os.stat(tree.LIB).st_mtime + 5
    os.utime(os.path.join(tree.CSRC, "calls.cpp"), (later, later))
    with pytest.raises(RuntimeError, match="calls.cpp"):
        tree.build()
    assert os.path.exists(tree.LIB) and not os.path.exists(os.path.join(tree.LIBDIR, tree.CALLS))


def test_without_pytorch_there_is_a_library(tree, monkeypatch):
    def missing(*_):
        raise ImportError("no torch")
    monkeypatch.setattr(tree, "_calls_commands", missing)
    with pytest.raises(RuntimeError, match="calls.cpp"):
        tree.build()
    assert os.path.exists(tree.LIB)


def test_nothing_is_built_twice(tree):
    tree.build()
    first = times(tree)
    assert tree.build() == tree.LIB and times(tree) == first


def test_another_pytorch_gets_another_module(tree, monkeypatch):
    import importlib.metadata
    tree.build()
    lib, calls = times(tree)
    monkeypatch.setattr(importlib.metadata, "version", lambda name: "0.0.1")
    tree.build()
    again = times(tree)
    assert again[0] == lib and again[1] > calls
    tree.build()
    assert times(tree) == again


def test_a_source_of_the_library_rebuilds_it(tree):
    tree.build()
    lib, _ = times(tree)
    later = os.stat(tree.LIB).st_mtime + 5
    os.utime(os.path.join(tree.CSRC, "one.cu"), (later, later))
    tree.build()
    assert times(tree)[0] > lib
