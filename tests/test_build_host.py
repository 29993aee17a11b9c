"""The library is built and serves where the Python entry of the decode-side calls cannot be; the entry is never an old one.
Nothing is compiled here: the library is there, and the entry's compiler is a stand-in."""
import os
import stat
import sys

import pytest

from paper_2505_19578_b200 import binding, build


@pytest.fixture
def calls(monkeypatch, tmp_path):
    """The entry's path for the test, with an entry of another torch in it."""
    build.build()
    path = str(tmp_path / "_decode_calls.so")
    with open(path, "wb") as f:
        f.write(b"shareprefill calls for torch 0.0.0, Python 2.7;")
    monkeypatch.setattr(build, "CALLS", path)
    return path


def compiler(tmp_path, body):
    path = str(tmp_path / "c++")
    with open(path, "w") as f:
        f.write("#!/bin/sh\n" + body)
    os.chmod(path, os.stat(path).st_mode | stat.S_IXUSR)
    return path


def test_without_torch_the_library_is_built(monkeypatch, calls):
    monkeypatch.setitem(sys.modules, "torch", None)
    monkeypatch.setenv("CXX", "/nowhere")
    assert build.build() == build.LIB and not build.calls_match(calls)


@pytest.mark.parametrize("there", [True, False])
def test_a_compiler_that_fails_leaves_no_entry_and_the_library(monkeypatch, calls, tmp_path, capsys, there):
    monkeypatch.setenv("CXX", compiler(tmp_path, "echo no headers; exit 1\n") if there else "/nowhere/c++")
    assert build.build() == build.LIB and not os.path.exists(calls)
    assert ("no headers" if there else "/nowhere/c++") in capsys.readouterr().err


def test_an_entry_of_another_torch_is_built_again(monkeypatch, calls, tmp_path):
    # writes what it was given into the file after -o
    monkeypatch.setenv("CXX", compiler(tmp_path, 'all="$*"\nwhile [ "$1" != -o ]; do shift; done\nprintf "%s" "$all" > "$2"\n'))
    assert build.calls_need_build()
    build.build()
    assert build.calls_match(calls) and not build.calls_need_build()


def test_the_headers_are_those_of_the_compiler(monkeypatch, calls, tmp_path):
    bin_dir = tmp_path / "toolkit" / "bin"
    bin_dir.mkdir(parents=True)
    nvcc = bin_dir / "nvcc"
    nvcc.write_text("#!/bin/sh\n")
    nvcc.chmod(0o755)
    monkeypatch.setenv("NVCC", str(nvcc))
    given = []
    monkeypatch.setattr(build.subprocess, "Popen", lambda cmd, **kw: given.append(cmd))
    build._start_calls_build()
    assert str(tmp_path / "toolkit" / "include") in given[0]


def test_an_entry_of_another_torch_is_not_loaded(monkeypatch, calls):
    monkeypatch.setattr(binding, "_native", None)
    monkeypatch.setattr(binding, "_HERE", os.path.dirname(calls))
    with pytest.raises(RuntimeError, match="another torch"):
        binding._decode_calls()
