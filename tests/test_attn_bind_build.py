"""The compiled part of the binding where it cannot be built, or was built for another torch: the library and every other call are there,
the calls that need it say so."""
import os
import sys
import types

import pytest
import torch

import paper_2608_22643_b200 as package
from paper_2608_22643_b200 import binding as nb
from paper_2608_22643_b200 import build as nbuild


@pytest.fixture()
def elsewhere(tmp_path, monkeypatch):
    """A binding to be built beside the real one, with an older one in its place."""
    nbuild.build()
    path = tmp_path / "np_attn_bind.so"
    path.write_bytes(b"of another day")
    os.utime(path, (1, 1))
    monkeypatch.setattr(nbuild, "BIND_PATH", str(path))
    return path


def _builds_without_it(path):
    with pytest.warns(UserWarning, match="np_attn_bind"):
        assert nbuild.build() == nbuild.LIB_PATH and os.path.exists(nbuild.LIB_PATH)
    assert not path.exists()                     # what was there is not of these sources
    assert nb.load() is not None
    with pytest.raises(nb.NpError):              # a call that goes through ctypes
        nb.np_kv_sizes(nb.make_kv_desc(torch.bfloat16, 0, 1, 64, 16, 1, 1))


def test_headers_are_missing(elsewhere, tmp_path, monkeypatch):
    source = tmp_path / "np_attn_bind.cpp"
    source.write_text("#include <no_such_header_anywhere.h>\n")
    monkeypatch.setattr(nbuild, "BIND_SOURCE", str(source))
    _builds_without_it(elsewhere)


def test_there_is_no_compiler(elsewhere, tmp_path, monkeypatch):
    monkeypatch.setenv("PATH", str(tmp_path))
    monkeypatch.setattr(nbuild, "_nvcc", lambda: "/usr/local/cuda/bin/nvcc")
    _builds_without_it(elsewhere)


def test_there_is_no_torch(elsewhere, monkeypatch):
    monkeypatch.setitem(sys.modules, "torch", None)
    _builds_without_it(elsewhere)


def test_the_calls_refuse_without_it(monkeypatch):
    nbuild.build()
    monkeypatch.setattr(nb, "_calls", None)
    monkeypatch.setitem(sys.modules, package.__name__ + ".np_attn_bind", None)
    monkeypatch.delattr(package, "np_attn_bind", raising=False)
    with pytest.raises(RuntimeError, match="np_attn_bind.so is not usable"):
        nb.np_kv_reset(None, None)


def test_the_calls_refuse_one_that_was_built_for_another_torch(monkeypatch):
    nbuild.build()
    monkeypatch.setattr(nb, "_calls", None)
    other = types.ModuleType(package.__name__ + ".np_attn_bind")
    other.built_for = "torch 1.0, python 3"
    monkeypatch.setitem(sys.modules, other.__name__, other)
    monkeypatch.setattr(package, "np_attn_bind", other, raising=False)
    with pytest.raises(RuntimeError, match="torch 1.0.*" + torch.__version__.replace("+", ".")):
        nb.np_kv_reset(None, None)
    assert nb._calls is None


def test_the_one_that_is_there_is_for_this_torch():
    nbuild.build()
    assert nb._attn().built_for == nbuild.bind_target()
