"""CPU-only: what an incremental build of the library compiles again (a stand-in for the compiler writes down what it was called for)."""
import os

import pytest

from paper_2408_10746_amd import build

COMPILER = """#!/bin/sh
echo "$@" >> "{log}"
while [ $# -gt 0 ]; do [ "$1" = -o ] && touch "$2"; shift; done
"""


@pytest.fixture
def tree(tmp_path, monkeypatch):
    csrc = tmp_path / "csrc"
    csrc.mkdir()
    for name in ("one.hip", "two.hip", "all.h"):
        (csrc / name).write_text("")
        os.utime(csrc / name, (1, 1))
    log, cc = tmp_path / "log", tmp_path / "cc"
    cc.write_text(COMPILER.format(log=log))
    cc.chmod(0o755)
    for name, value in dict(CSRC=str(csrc), LIB=str(tmp_path / "lib.so"), OBJ_DIR=str(tmp_path / "obj"), SOURCES=["one.hip", "two.hip"], HEADERS=["all.h"],
                            HIPCC_FLAGS=["-a"], SOURCE_FLAGS={"two.hip": ["-b"]}).items():
        monkeypatch.setattr(build, name, value)
    monkeypatch.setenv("HIPCC", str(cc))

    def made(force=False):
        log.write_text("")
        build.build_lib(force)
        lines = log.read_text().splitlines()
        return sorted(w[:-4] for line in lines for w in [line.split()[-1].rsplit("/")[-1]] if w.endswith(".hip")), sum("-shared" in line for line in lines)

    return csrc, made


def test_what_is_compiled_again(tree, monkeypatch):
    csrc, made = tree
    assert made() == (["one", "two"], 1) and made() == ([], 0)
    os.utime(csrc / "one.hip")
    os.utime(csrc / "one.hip", (os.path.getmtime(csrc / "one.hip") + 5,) * 2)
    assert made() == (["one"], 1)
    assert made(True) == (["one", "two"], 1)


def test_changed_flags_make_objects_again(tree, monkeypatch):
    csrc, made = tree
    made()
    monkeypatch.setattr(build, "SOURCE_FLAGS", {"two.hip": ["-c2"]})
    assert made() == (["two"], 1) and made() == ([], 0)
    monkeypatch.setattr(build, "SOURCE_FLAGS", {})
    assert made() == (["two"], 1) and made() == ([], 0)
    monkeypatch.setattr(build, "HIPCC_FLAGS", ["-a", "-d"])
    assert made() == (["one", "two"], 1) and made() == ([], 0)


def test_a_library_that_was_not_linked_is_linked(tree, monkeypatch):
    """Objects made, then the link fails: the old library does not pass for the new one."""
    csrc, made = tree
    made()
    os.utime(build.LIB, (2, 2))
    assert made() == ([], 1)
