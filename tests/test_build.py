"""The build without a GPU: the C library does not depend on what only its Python binding needs."""

import os

import pytest

from paper_2605_06892_amd import build as B


@pytest.fixture
def small(monkeypatch, tmp_path):
    """A library of one empty source, in a folder of its own, with a binding left by an earlier build."""
    src = tmp_path / "csrc"
    src.mkdir()
    (src / "one.hip").write_text('extern "C" __attribute__((visibility("default"))) int one() { return 1; }\n')
    for name, path in (("CSRC", src), ("OBJ", tmp_path / "obj"), ("LIB", tmp_path / "lib.so"), ("BINDING", tmp_path / "b.so")):
        monkeypatch.setattr(B, name, str(path))
    (tmp_path / "b.so").write_text("stale")
    return tmp_path


@pytest.mark.parametrize("step", ["_compile_binding", "_link_binding"])
@pytest.mark.parametrize("error", [RuntimeError, FileNotFoundError, ImportError])
def test_library_without_binding(small, monkeypatch, step, error):
    """No host compiler, or no headers of torch: the library is there, the build says what is not, and a binding of an
    older library is gone."""
    def fail(*_):
        raise error("no such tool")

    monkeypatch.setattr(B, "_compile_binding", lambda: "obj")
    monkeypatch.setattr(B, step, fail)
    with pytest.raises(RuntimeError, match="binding.*no such tool"):
        B.build()
    assert os.path.exists(B.LIB) and not os.path.exists(B.BINDING)


def test_library_that_does_not_compile(small, monkeypatch):
    monkeypatch.setattr(B, "_compile_binding", lambda: "obj")
    (small / "csrc" / "two.hip").write_text("not C++")
    with pytest.raises(RuntimeError, match="two.hip"):
        B.build()
    assert not os.path.exists(B.LIB)
