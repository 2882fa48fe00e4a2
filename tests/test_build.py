"""CPU checks of the build itself: the C library needs hipcc only; what calls it from torch tensors is built beside it."""
import os
import stat
import sys

import pytest

from paper_2308_15949_amd import build


@pytest.fixture
def compiler(tmp_path, monkeypatch):
    """A stand-in for hipcc that makes the file it is asked for, and a tree of its own for what is made."""
    script = tmp_path / "cc"
    script.write_text('#!/bin/sh\nwhile [ $# -gt 0 ]; do [ "$1" = -o ] && { shift; : > "$1"; }; shift; done\n')
    script.chmod(script.stat().st_mode | stat.S_IXUSR)
    monkeypatch.setenv("HIPCC", str(script))
    for name, path in (("OBJ", "obj"), ("LIB", "liblaud.so"), ("EXTENSION", "_laud_torch.so")):
        monkeypatch.setattr(build, name, str(tmp_path / path))
    return str(script)


def test_the_library_is_built_where_there_is_no_torch(compiler, monkeypatch, capsys):
    monkeypatch.setitem(sys.modules, "torch", None)  # (importing it raises ImportError)
    assert build.build(verbose=False) == build.LIB and os.path.exists(build.LIB)
    assert not os.path.exists(build.EXTENSION)
    assert "torch" in capsys.readouterr().err  # said, not silent


def test_the_library_is_built_where_the_extension_fails(compiler, monkeypatch):
    monkeypatch.setenv("CXX", "/bin/false")
    with pytest.raises(RuntimeError, match="false"):
        build.build(verbose=False)
    assert os.path.exists(build.LIB)


def test_a_source_that_fails_is_an_error(compiler, monkeypatch):
    monkeypatch.setenv("HIPCC", "/bin/false")
    monkeypatch.setenv("CXX", compiler)
    with pytest.raises(RuntimeError, match="false"):
        build.build(verbose=False)
    assert not os.path.exists(build.LIB)


def test_both_are_built(compiler, monkeypatch):
    monkeypatch.setenv("CXX", compiler)
    build.build(verbose=False)
    assert os.path.exists(build.LIB) and os.path.exists(build.EXTENSION)


def test_the_extension_is_compiled_as_torch_was(monkeypatch, tmp_path):
    import torch
    monkeypatch.setenv("ROCM_PATH", str(tmp_path))
    command = build.extension_command()
    assert f"-D_GLIBCXX_USE_CXX11_ABI={int(torch.compiled_with_cxx11_abi())}" in command
    assert str(tmp_path / "include") in command
