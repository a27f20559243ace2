"""The build on hosts that lack what only the binding's native part takes (CPU)."""

import os
import sysconfig

import pytest

from paper_1511_05946_amd import build as B


@pytest.fixture
def made(monkeypatch, tmp_path):
    """build() without hipcc, and an older binding where its own would go."""
    lib = tmp_path / "libacdc.so"

    def library(verbose=False, extra_flags=None):
        lib.write_bytes(b"")
        return str(lib)

    monkeypatch.setattr(B, "build_library", library, raising=False)
    monkeypatch.setattr(B, "hipcc", lambda: pytest.fail("the library is not what is tested"))
    monkeypatch.setattr(B, "LIB", str(lib))
    monkeypatch.setattr(B, "BINDING", str(tmp_path / "_train_binding.so"))
    (tmp_path / "_train_binding.so").write_bytes(b"old")
    return lib


def test_library_without_a_host_compiler(made, monkeypatch, capsys):
    monkeypatch.setenv("CXX", "no-such-compiler")
    assert B.build() == str(made) and made.exists()
    assert not os.path.exists(B.BINDING)   # not an older library's
    assert "g++" in capsys.readouterr().err
    with pytest.raises(RuntimeError, match="g\\+\\+"):
        B.build_binding()


def test_library_without_pythons_headers(made, monkeypatch, capsys, tmp_path):
    monkeypatch.setattr(sysconfig, "get_paths", lambda: {"include": str(tmp_path)})
    assert B.build() == str(made)
    assert "Python.h" in capsys.readouterr().err


def test_library_without_torch(made, monkeypatch, capsys):
    import importlib.util
    find = importlib.util.find_spec
    monkeypatch.setattr(importlib.util, "find_spec", lambda name, *a: None if name == "torch" else find(name, *a))
    assert B.build() == str(made)
    assert "no torch" in capsys.readouterr().err


def test_binding_that_does_not_compile_is_an_error(made, monkeypatch, capsys):
    monkeypatch.setenv("CXX", "false")
    if B.missing_for_binding() is not None:
        pytest.skip("no headers or torch here")
    with pytest.raises(RuntimeError, match="failed"):
        B.build()
