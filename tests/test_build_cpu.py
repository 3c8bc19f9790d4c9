"""What building does where only part of it can be built."""
import os

import pytest

from paper_2310_11453_b200 import build as bl_build


@pytest.fixture
def sandbox(tmp_path, monkeypatch):
    """The build in a folder of its own, with a compiler that only notes its calls and makes empty files."""
    log, nvcc = tmp_path / "log", tmp_path / "nvcc"
    nvcc.write_text(f'#!/bin/sh\necho "$@" >> {log}\nwhile [ $# -gt 1 ]; do [ "$1" = -o ] && : > "$2"; shift; done\n')
    nvcc.chmod(0o755)
    for name, value in (("NVCC", nvcc), ("LIB", tmp_path / "lib.so"), ("MARSHAL", tmp_path / "marshal.so"), ("OBJ", tmp_path / "obj")):
        monkeypatch.setattr(bl_build, name, str(value))
    return tmp_path, lambda: len(log.read_text().splitlines()) if log.exists() else 0


@pytest.mark.parametrize("cxx", ["false", "/no/such/compiler"])
def test_the_library_is_built_where_the_marshalling_cannot_be(sandbox, monkeypatch, capsys, cxx):
    path, calls = sandbox
    monkeypatch.setenv("CXX", cxx)
    (path / "marshal.so").write_text("of an earlier build")
    assert bl_build.build(force=True) == str(path / "lib.so") and (path / "lib.so").exists()
    assert not (path / "marshal.so").exists() and "no attention operators" in capsys.readouterr().err
    n = calls()
    assert n == len(bl_build.sources()) + 1
    assert bl_build.build() == str(path / "lib.so") and calls() == n      # the library is not built again for it
    os.utime(path / "lib.so", (0, 0))
    bl_build.build()
    assert calls() == 2 * n


def test_a_library_that_does_not_compile_is_an_error(sandbox, monkeypatch):
    monkeypatch.setenv("CXX", "false")
    monkeypatch.setattr(bl_build, "NVCC", "false")
    with pytest.raises(RuntimeError):
        bl_build.build(force=True)
