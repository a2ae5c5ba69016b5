"""The library builds without what only the operators' Python binding needs
(torch's headers and a C++ compiler of the host); a binding that is there is
never one of another build.  CPU only."""
import os

import pytest

from paper_2111_05426_amd import build


@pytest.fixture
def elsewhere(monkeypatch, tmp_path):
    """build() with the library's compilation replaced and the binding in tmp_path."""
    ran = []
    monkeypatch.setattr(build, "_build_library", lambda hipcc, verbose: ran.append("library"))
    monkeypatch.setattr(build, "BINDING", str(tmp_path / "_ops.so"))
    (tmp_path / "_ops.so").write_text("of another build")
    return ran, tmp_path


def test_without_a_compiler(elsewhere, monkeypatch, capsys):
    ran, tmp = elsewhere
    monkeypatch.setenv("CXX", str(tmp / "no-such-compiler"))
    assert build.build() == build.LIB and ran == ["library"]
    assert os.listdir(tmp) == [] and "no-such-compiler" in capsys.readouterr().err


@pytest.mark.parametrize("root", [None, "empty"])
def test_without_torch_headers(elsewhere, monkeypatch, capsys, root):
    ran, tmp = elsewhere
    monkeypatch.setattr(build, "_torch_root", lambda: root and str(tmp / root))
    assert build.build() == build.LIB and ran == ["library"]
    assert os.listdir(tmp) == [] and "torch" in capsys.readouterr().err


def test_what_does_not_compile_is_an_error(elsewhere, monkeypatch):
    _, tmp = elsewhere
    source = tmp / "broken.cpp"
    source.write_text("#error broken\n")
    monkeypatch.setattr(build, "binding_sources", lambda: [str(source)])
    with pytest.raises(Exception):
        build.build()
