"""The C library is built with hipcc alone: without torch, Python's headers or a host compiler it is there, and what is missing
is said."""
import os
import sys

import pytest

from paper_2603_08957_amd import build


@pytest.fixture
def small(monkeypatch, tmp_path):
    """A build of one of the library's sources into a folder of its own."""
    monkeypatch.setattr(build, "OBJ", str(tmp_path / "obj"))
    monkeypatch.setattr(build, "LIB", str(tmp_path / "libtre.so"))
    monkeypatch.setattr(build, "TENSORS", str(tmp_path / "_tensors.so"))
    monkeypatch.setattr(build, "sources", lambda: [os.path.join(build.CSRC, "events.cpp")])
    return tmp_path


def test_without_torch(small, monkeypatch, capsys):
    monkeypatch.setitem(sys.modules, "torch", None)
    assert build.build() == build.LIB
    assert os.path.exists(build.LIB) and not os.path.exists(build.TENSORS)
    assert "_tensors.so" in capsys.readouterr().err


@pytest.mark.parametrize("compiler", ["no-such-compiler", "false"])
def test_without_a_host_compiler(small, monkeypatch, compiler):
    """The library is there; a binding that cannot be built where torch is there is an error."""
    monkeypatch.setenv("CXX", compiler)
    with pytest.raises(RuntimeError, match="_tensors.so|tensors.cpp"):
        build.build()
    assert os.path.exists(build.LIB) and not os.path.exists(build.TENSORS)


def test_library_alone(small, monkeypatch):
    monkeypatch.setattr(build, "build_tensors", lambda: pytest.fail("asked for"))
    assert build.build(binding=False) == build.LIB and os.path.exists(build.LIB)


def test_a_source_that_does_not_compile(small, monkeypatch):
    (small / "bad.cpp").write_text("not C++")
    monkeypatch.setattr(build, "sources", lambda: [str(small / "bad.cpp")])
    monkeypatch.setattr(build, "build_tensors", lambda: None)
    with pytest.raises(RuntimeError, match="bad.cpp"):
        build.build()
    assert not os.path.exists(build.LIB)
