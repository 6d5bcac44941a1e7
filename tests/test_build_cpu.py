"""The build's decisions about the extension module, in a folder of its own (no nvcc, no GPU)."""
import os
import sysconfig

import pytest

from paper_2609_38767_gb300 import build as tbuild


@pytest.fixture
def folder(tmp_path, monkeypatch):
    monkeypatch.setattr(tbuild, "lib_path", lambda name: str(tmp_path / name))
    monkeypatch.setattr(tbuild, "BUILD", str(tmp_path))
    return tmp_path


def test_the_extension_is_built_for_the_python_that_asks(folder, monkeypatch):
    """A module left by another Python has another ABI; its file's age says nothing about that."""
    target = tbuild.build_fast()
    first = os.stat(target).st_mtime_ns
    assert tbuild.build_fast() == target and os.stat(target).st_mtime_ns == first  # up to date: left alone
    real = sysconfig.get_config_var
    monkeypatch.setattr(tbuild.sysconfig, "get_config_var", lambda k: "cpython-399-other" if k == "SOABI" else real(k))
    tbuild.build_fast()
    second = os.stat(target).st_mtime_ns
    assert second != first
    tbuild.build_fast()
    assert os.stat(target).st_mtime_ns == second


def test_without_pythons_headers_the_rest_is_built(folder, monkeypatch):
    """Attribution alone needs no extension module: its build goes through and says what is missing."""
    monkeypatch.setattr(tbuild, "LIBS", {})
    monkeypatch.setattr(tbuild, "build_synth_cpu", lambda: "synth")
    paths = dict(sysconfig.get_paths(), include=str(folder / "none"))
    monkeypatch.setattr(tbuild.sysconfig, "get_paths", lambda *a, **k: paths)
    with pytest.warns(UserWarning, match="Python.h"):
        out = tbuild.build()
    assert out == {"libtda_synth_cpu.so": "synth"} and not (folder / "_fast.so").exists()
