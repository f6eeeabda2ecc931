"""The library builds where the binding's headers or compiler are not installed; a binding that does not compile
fails the build.  Host only; the library itself is not compiled here."""
import shutil

import pytest

from paper_1702_07005_amd import build


@pytest.fixture
def no_library(monkeypatch, tmp_path):
    monkeypatch.setattr(build, "_compile", lambda sources, out, verbose: out)
    monkeypatch.setattr(build, "BINDING", str(tmp_path / "_features.so"))
    return tmp_path


@pytest.mark.parametrize("lack", ["Python.h", "torch", "g++", "torch/csrc"])
def test_library_builds_without_the_binding(no_library, monkeypatch, capsys, lack):
    import importlib.util
    import types
    (no_library / "_features.so").write_text("of another library")
    if lack == "Python.h":
        monkeypatch.setattr(build.sysconfig, "get_paths", lambda: {"include": str(no_library)})
    elif lack == "g++":
        monkeypatch.setattr(shutil, "which", lambda name: None)
    else:
        spec = None if lack == "torch" else types.SimpleNamespace(origin=str(no_library / "__init__.py"))
        monkeypatch.setattr(importlib.util, "find_spec", lambda name: spec)
    assert build.build() == build.LIB
    assert lack in capsys.readouterr().err and not (no_library / "_features.so").exists()


@pytest.mark.skipif(shutil.which("g++") is None, reason="needs g++")
def test_binding_that_does_not_compile_fails_the_build(no_library, monkeypatch):
    broken = no_library / "binding.cpp"
    broken.write_text("#error not this one\n")
    monkeypatch.setattr(build, "BINDING_SOURCE", str(broken))
    with pytest.raises(RuntimeError, match="g\\+\\+ failed"):
        build.build()
