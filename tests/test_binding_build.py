"""The short way from Python to the library is an extra: it fits one Python and one torch, and everything works without it.  Host only."""
import subprocess

import pytest
import torch


@pytest.fixture
def fresh(monkeypatch):
    """(build, gvq), the library built but not loaded."""
    from paper_1811_03617_b200 import build, gvq
    build.build()
    monkeypatch.setattr(gvq, "_lib", None)
    monkeypatch.setattr(gvq, "_short", None)
    return build, gvq


def test_the_library_loads_without_the_module(fresh, monkeypatch, tmp_path):
    build, gvq = fresh
    for content in (None, b"", b"not a shared library"):
        path = tmp_path / f"_binding.{content!r:.4}.so"
        if content is not None:
            path.write_bytes(content)
        monkeypatch.setattr(build, "binding_path", lambda: path)
        monkeypatch.setattr(gvq, "_lib", None)
        with pytest.warns(RuntimeWarning, match="ctypes"):
            L = gvq.lib()
        assert gvq._short is None and L.gvq_i8_codes_bytes(7, 33) == 7 * 48
        assert gvq.lib() is L


def test_the_library_is_wanted(fresh, monkeypatch, tmp_path):
    _, gvq = fresh
    monkeypatch.setattr(gvq, "LIB_PATH", tmp_path / "libgvq.so")
    with pytest.raises(RuntimeError, match="missing"):
        gvq.lib()


def test_the_module_is_loaded_where_it_fits(fresh, recwarn):
    _, gvq = fresh
    gvq.lib()
    assert gvq._short is not None and not [w for w in recwarn if "ctypes" in str(w.message)]


def test_another_torch_or_python_has_a_module_of_its_own(fresh, monkeypatch):
    import sysconfig
    build, _ = fresh
    mine = build.binding_path()
    assert mine.exists() and not build._stale_binding() and not build._stale()
    with monkeypatch.context() as m:
        m.setattr(torch, "__version__", "0.0.1")
        assert build.binding_path() != mine and build._stale_binding() and not build._stale()
    with monkeypatch.context() as m:
        m.setattr(sysconfig, "get_config_var", lambda name: "cpython-0")
        assert build.binding_path() != mine and build._stale_binding()


@pytest.mark.parametrize("command", [["false"], ["/nowhere/a-compiler"]])
def test_a_module_that_cannot_be_built_is_a_warning(fresh, monkeypatch, tmp_path, command):
    build, _ = fresh
    path = tmp_path / "_binding.so"
    monkeypatch.setattr(build, "binding_path", lambda: path)
    monkeypatch.setattr(build, "_binding_command", lambda out: command)
    with pytest.warns(RuntimeWarning, match="was not built"):
        assert build.build() == build.LIB
    assert list(tmp_path.iterdir()) == [] and build.LIB.exists()


def test_a_library_that_cannot_be_built_is_an_error(fresh, monkeypatch, tmp_path):
    build, _ = fresh
    monkeypatch.setattr(build, "LIB", tmp_path / "libgvq.so")
    monkeypatch.setattr(build, "NVCC_FLAGS", ["--no-such-flag"])
    with pytest.raises(subprocess.CalledProcessError):
        build.build()
    assert list(tmp_path.iterdir()) == []
