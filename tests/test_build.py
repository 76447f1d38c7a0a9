"""The library's build beside that of its Python side, which alone needs PyTorch and g++.  (Stand-in sources; no GPU.)"""
import ctypes as C
import os
import sys

import pytest

from paper_2011_06295_amd import build


@pytest.fixture
def sources(tmp_path, monkeypatch):
    """A library of one small source in a folder of its own."""
    (tmp_path / "one.cpp").write_text('extern "C" int answer() { return 42; }\n')
    (tmp_path / "text_torch.cpp").write_text('extern "C" int torch_side() { return 1; }\n')
    for name, value in {"CSRC": str(tmp_path), "SOURCES": ["one.cpp"], "LIB": str(tmp_path / "library.so"), "TORCH_LIB": str(tmp_path / "_torch.so")}.items():
        monkeypatch.setattr(build, name, value)
    return tmp_path


def _answer():
    return C.CDLL(build.LIB).answer()


def test_both_are_built(sources):
    assert build.build() == build.LIB
    assert _answer() == 42 and C.CDLL(build.TORCH_LIB).torch_side() == 1
    assert sorted(p.name for p in sources.iterdir()) == ["_torch.so", "library.so", "one.cpp", "text_torch.cpp"]


def test_the_library_needs_no_pytorch(sources, monkeypatch, capsys):
    monkeypatch.setitem(sys.modules, "torch", None)         # import torch raises ImportError
    assert build.build(verbose=True) == build.LIB
    assert _answer() == 42 and not os.path.exists(build.TORCH_LIB)
    assert "PyTorch" in capsys.readouterr().out


def test_the_library_is_linked_where_its_python_side_does_not_compile(sources):
    (sources / "text_torch.cpp").write_text("this is no C++\n")
    (sources / "_torch.so").write_text("the one that was there")
    with pytest.raises(RuntimeError, match=r"g\+\+ failed"):
        build.build()
    assert _answer() == 42 and (sources / "_torch.so").read_text() == "the one that was there"


def test_nothing_is_written_where_the_library_does_not_compile(sources):
    (sources / "one.cpp").write_text("this is no C++\n")
    with pytest.raises(RuntimeError, match="hipcc failed"):
        build.build()
    assert not os.path.exists(build.LIB)
