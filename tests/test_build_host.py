"""The build without what the binding's module needs: the library is made all the
same, with a warning, no module of other sources stays behind, and the calls that
need it say so.  The CUDA compiler is a stand-in that writes its output file."""
import importlib
import os
import sysconfig

import pytest

from paper_2607_11951_gb300 import grid as G

B = importlib.import_module("paper_2607_11951_gb300.build")


@pytest.fixture
def place(tmp_path, monkeypatch):
    nvcc = tmp_path / "bin" / "nvcc"
    nvcc.parent.mkdir()
    nvcc.write_text('#!/bin/sh\nwhile [ "$1" != -o ]; do shift; done\n: > "$2"\n')
    nvcc.chmod(0o755)
    out = tmp_path / "out"
    out.mkdir()
    monkeypatch.setattr(B, "OUT", str(out))
    monkeypatch.setattr(B, "NVCC", str(nvcc))
    (out / "grid_binding.so").write_text("of other sources")
    return tmp_path


def built_without(why):
    with pytest.warns(RuntimeWarning, match="grid_binding.so was not built") as w:
        path = B.build()
    assert path == B.library_path() and os.path.exists(path) and not os.path.exists(B.binding_path())
    assert why in str(w[0].message)


def test_no_compiler_for_the_module(place, monkeypatch):
    monkeypatch.setenv("PATH", str(place / "bin"))
    built_without("g++")


def test_no_headers(place, monkeypatch):
    empty = place / "empty"
    empty.mkdir()
    monkeypatch.setattr(sysconfig, "get_paths", lambda: {"include": str(empty)})
    monkeypatch.setattr(B, "CSRC", str(place))
    (place / "grid_python.cpp").write_text("#include <Python.h>\n")
    built_without("Python.h")


def test_no_torch(place, monkeypatch):
    monkeypatch.setattr(importlib.util, "find_spec", lambda name: None)
    built_without("torch")


def test_a_symbol_that_does_not_resolve(place, monkeypatch):
    """The linker leaves it to the loader; the build loads the module."""
    monkeypatch.setattr(B, "CSRC", str(place))
    (place / "grid_python.cpp").write_text('extern "C" void* nowhere();\nextern "C" void* PyInit_grid_binding() { return nowhere(); }\n')
    built_without("nowhere")


def test_a_failing_library_is_an_error(place, monkeypatch):
    (place / "bin" / "nvcc").write_text("#!/bin/sh\nexit 1\n")
    monkeypatch.setattr(B, "build_binding", lambda: None)
    with pytest.raises(RuntimeError, match="nvcc failed"):
        B.build()


def test_calls_that_need_the_module_say_so(place, monkeypatch):
    monkeypatch.setattr(G, "_calls", None)
    monkeypatch.setattr(G, "binding_path", lambda: str(place / "none.so"))
    with pytest.raises(G.GridLibraryMissing, match="grid_binding.so"):
        G.grid_tree_plan(None, None, None, None)
