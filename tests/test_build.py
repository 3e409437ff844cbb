"""The library is built with nvcc alone; only the tensor front end needs PyTorch."""
import os

import pytest

from paper_2110_06037_gb300 import build as b


@pytest.fixture
def steps(tmp_path, monkeypatch):
    """What a build from nothing does, with the compilers left out."""
    done = []
    monkeypatch.setattr(b, "BUILD", str(tmp_path / "build"))
    monkeypatch.setattr(b, "LIB", str(tmp_path / "libsn.so"))
    monkeypatch.setattr(b, "BIND", str(tmp_path / "_blocks.so"))
    monkeypatch.setattr(b, "_compile", lambda src, verbose: os.path.basename(src))
    monkeypatch.setattr(b, "_link", lambda objs: done.append("libsn"))
    monkeypatch.setattr(b, "_link_bind", lambda obj: done.append("front end"))
    return done


def test_without_pytorch_the_library_is_built(steps, monkeypatch):
    find = b.importlib.util.find_spec
    monkeypatch.setattr(b.importlib.util, "find_spec", lambda name: None if name == "torch" else find(name))
    assert b.build() == b.LIB
    assert steps == ["libsn"]


def test_a_front_end_that_does_not_compile_leaves_the_library(steps, monkeypatch):
    def broken():
        raise RuntimeError("no such header")

    monkeypatch.setattr(b, "_compile_bind", broken)
    with pytest.raises(RuntimeError, match="no such header"):
        b.build()
    assert steps == ["libsn"]


def test_with_pytorch_both_are_built_the_library_first(steps, monkeypatch):
    monkeypatch.setattr(b, "_compile_bind", lambda: "bind")
    b.build()
    assert steps == ["libsn", "front end"]
