"""The build installs each of its two files when it is made (compilers stand in; no GPU)."""
import os
import stat

import pytest

from paper_2607_26005_amd import build

COMPILER = """#!/bin/sh
while [ $# -gt 0 ]; do if [ "$1" = -o ]; then echo %s > "$2"; fi; shift; done
exit %d
"""


@pytest.fixture
def stand_ins(tmp_path, monkeypatch):
    def make(name, code=0):
        p = tmp_path / name
        p.write_text(COMPILER % (name, code))
        p.chmod(p.stat().st_mode | stat.S_IEXEC)
        return str(p)
    monkeypatch.setattr(build, "LIB", str(tmp_path / "libpictura.so"))
    monkeypatch.setattr(build, "TENSORS", str(tmp_path / "_tensors.so"))
    monkeypatch.setattr(build, "CSRC", str(tmp_path))
    monkeypatch.setenv("HIPCC", make("hipcc"))
    monkeypatch.setenv("CXX", make("c++"))
    return make


def test_both_files_are_installed(stand_ins):
    assert build.build() == build.LIB
    assert open(build.LIB).read() == "hipcc\n" and open(build.TENSORS).read() == "c++\n"


@pytest.mark.parametrize("why", ["no compiler", "compiler fails", "no torch"])
def test_the_library_is_there_where_the_helper_cannot_be_built(stand_ins, monkeypatch, why):
    if why == "no torch":
        import sys
        monkeypatch.setitem(sys.modules, "torch", None)
    else:
        monkeypatch.setenv("CXX", "/nowhere/c++" if why == "no compiler" else stand_ins("broken", 1))
    with pytest.raises(RuntimeError, match="_tensors.so, which the policy's operators need, is not"):
        build.build()
    assert open(build.LIB).read() == "hipcc\n" and not os.path.exists(build.TENSORS)


def test_a_library_that_cannot_be_built_replaces_nothing(stand_ins, monkeypatch):
    open(build.LIB, "w").write("before\n")
    monkeypatch.setenv("HIPCC", stand_ins("broken", 1))
    with pytest.raises(RuntimeError, match="broken failed"):
        build.build()
    assert open(build.LIB).read() == "before\n"
