"""The library builds with hipcc alone; Python's side of it needs torch as well, and is built where torch is."""
import os
import stat

import pytest

from paper_1503_05032_amd import build as libbuild


@pytest.fixture
def elsewhere(tmp_path, monkeypatch):
    """Builds go to a folder of their own, by a compiler that writes empty files and notes what it was asked for."""
    fake = tmp_path / "compiler"
    fake.write_text('#!/bin/sh\necho "$@" >> "$(dirname "$0")/asked"\nwhile [ $# -gt 1 ]; do [ "$1" = -o ] && : > "$2"; shift; done\n')
    fake.chmod(fake.stat().st_mode | stat.S_IXUSR)
    for name, value in (("HIPCC", str(fake)), ("CXX", str(fake))):
        monkeypatch.setenv(name, value)
    monkeypatch.setattr(libbuild, "OUT", str(tmp_path / "libcsr5.so"))
    monkeypatch.setattr(libbuild, "MARSHAL", str(tmp_path / "_marshal.so"))
    return tmp_path


def test_without_torch_the_library_alone_is_built(elsewhere, monkeypatch):
    real = libbuild.importlib.util.find_spec
    monkeypatch.setattr(libbuild.importlib.util, "find_spec", lambda name, *a: None if name == "torch" else real(name, *a))
    assert libbuild.is_stale()
    assert libbuild.build(verbose=False) == libbuild.OUT
    assert os.path.exists(libbuild.OUT) and not os.path.exists(libbuild.MARSHAL)
    assert not libbuild.is_stale()
    assert "marshal.cpp" not in (elsewhere / "asked").read_text()


def test_with_torch_both_are_built(elsewhere):
    assert libbuild.is_stale()
    libbuild.build(verbose=False)
    assert os.path.exists(libbuild.OUT) and os.path.exists(libbuild.MARSHAL)
    assert not libbuild.is_stale()
    os.utime(libbuild.MARSHAL, (1, 1))
    assert libbuild.is_stale()


def test_a_host_compiler_is_found_without_gxx(monkeypatch):
    monkeypatch.delenv("CXX", raising=False)
    real = libbuild.shutil.which
    monkeypatch.setattr(libbuild.shutil, "which", lambda c, *a, **k: None if c == "g++" else real(c, *a, **k))
    assert os.path.basename(libbuild.host_compiler()).startswith("clang++")
