"""The extension with the cache's calls is optional: a build where it does not compile goes on without it.  No GPU."""
import os
import subprocess
import sys

import pytest

from paper_2608_01655_gb300 import build as ppbuild

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


@pytest.fixture
def place(tmp_path, monkeypatch):
    """A module's place, source and compiler of their own; the library is built."""
    ppbuild.build()
    if not ppbuild._python_include():
        pytest.skip("no Python headers")
    lib, src, bin_ = tmp_path / "_pp_call.so", tmp_path / "pp_call.c", tmp_path / "bin"
    src.write_text(open(ppbuild.CALL_SRC).read())
    bin_.mkdir()
    monkeypatch.setattr(ppbuild, "CALL_LIB", str(lib))
    monkeypatch.setattr(ppbuild, "CALL_SRC", str(src))
    return lib, src, bin_


def test_a_source_that_does_not_compile(place):
    lib, src, _ = place
    src.write_text("#include <Python.h>\nint f(void) { return no_such_call(; }\n")
    with pytest.warns(UserWarning, match="ctypes"):
        assert ppbuild.build() == ppbuild.LIB
    assert not lib.exists() and os.listdir(lib.parent).count("_pp_call.so") == 0
    assert not [f for f in os.listdir(lib.parent) if ".tmp" in f]


def test_one_that_is_out_of_date_does_not_stay(place):
    """A module of older sources could have other arguments than the library."""
    lib, src, _ = place
    lib.write_text("")
    os.utime(lib, (1, 1))
    src.write_text("#error older\n")
    with pytest.warns(UserWarning, match="older"):
        ppbuild.build()
    assert not lib.exists()


def test_no_compiler(place, monkeypatch):
    lib, _, bin_ = place
    monkeypatch.setenv("PATH", str(bin_))
    with pytest.warns(UserWarning, match="ctypes"):
        assert ppbuild.build() == ppbuild.LIB
    assert not lib.exists()


def test_a_compiler_that_fails(place, monkeypatch):
    lib, _, bin_ = place
    gcc = bin_ / "gcc"
    gcc.write_text("#!/bin/sh\necho broken >&2\nexit 1\n")
    gcc.chmod(0o755)
    monkeypatch.setenv("PATH", f"{bin_}:{os.environ['PATH']}")
    with pytest.warns(UserWarning, match="broken"):
        ppbuild.build()
    assert not lib.exists()


def test_it_is_built_once_and_again_when_its_source_is_newer(place):
    lib, src, _ = place
    ppbuild.build()
    first = lib.stat().st_mtime_ns
    ppbuild.build()
    assert lib.stat().st_mtime_ns == first
    os.utime(lib, (1, 1))
    ppbuild.build()
    assert lib.stat().st_mtime > 1


def test_without_headers_there_is_none(place, monkeypatch):
    lib, _, _ = place
    monkeypatch.setattr(ppbuild, "_python_include", lambda: None)
    ppbuild.build()
    assert not lib.exists()


def test_the_binding_does_without():
    ppbuild.build()
    code = ("import sys; sys.modules['paper_2608_01655_gb300._pp_call'] = None\n"
            "from paper_2608_01655_gb300 import binding as pp\n"
            "assert pp._fast is None and pp._lib.pp_kv_sync(None, None) == pp.PP_EINVAL\n"
            "assert pp._lib.pp_kv_write(None, 0, None, 0, 0, None, 0, 0, None, None, None, None) == pp.PP_EINVAL\n")
    subprocess.run([sys.executable, "-c", code], check=True, cwd=ROOT)
