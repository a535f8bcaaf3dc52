"""The build makes again what was made from other sources or by another command, and nothing else (compilers that only note how they were
called; no CUDA code is compiled here)."""
import os
import sys

import pytest
import torch

from paper_2602_02071_b200 import build

COMPILER = """#!/bin/sh
echo "$@" >> "$(dirname "$0")/calls"
case "$*" in *fail.cu*) exit 1;; esac
while [ "$1" != "-o" ]; do shift; done
echo "made" > "$2"
"""


class Tree:
    def __init__(self, d, monkeypatch):
        self.d, self.monkeypatch = d, monkeypatch
        for name, text in (("a.cu", '#include "both.cuh"\n'), ("b.cu", '#include "both.cuh"\n'), ("both.cuh", ""), ("serving_marshal.cpp", "")):
            (d / name).write_text(text)
        for name in ("nvcc", "other_nvcc", "cxx"):
            (d / name).write_text(COMPILER)
            (d / name).chmod(0o755)
        monkeypatch.setattr(build, "CSRC", str(d))
        monkeypatch.setattr(build, "UNITS", ["a.cu", "b.cu"])
        monkeypatch.setattr(build, "MARSHAL", str(d / "marshal.so"))
        monkeypatch.setenv("NVCC", str(d / "nvcc"))
        monkeypatch.setenv("CXX", str(d / "cxx"))

    def count(self, fn):
        calls = self.d / "calls"
        calls.write_text("")
        fn()
        return len(calls.read_text().splitlines())

    def library(self, *flags):
        return self.count(lambda: build._compile(str(self.d / "lib.so"), list(flags), str(self.d / "lib.log"), False, False))

    def marshal(self):
        return self.count(lambda: build._compile_marshal(False))

    def age(self):
        """All files but the sources are a minute older than now."""
        for p in self.d.iterdir():
            os.utime(p, (os.path.getmtime(p) - 60,) * 2)

    def touch(self, name):
        os.utime(self.d / name)


@pytest.fixture
def tree(tmp_path, monkeypatch):
    return Tree(tmp_path, monkeypatch)


def test_what_is_current_is_not_made_again(tree):
    assert tree.library() == 3 and tree.library() == 0             # two units and the link
    tree.age()
    tree.touch("b.cu")
    assert tree.library() == 2 and tree.library() == 0
    tree.age()
    tree.touch("both.cuh")
    assert tree.library() == 3


def test_other_flags_or_another_compiler_make_everything_again(tree):
    assert tree.library() == 3
    assert tree.library("-DX=1") == 3 and tree.library("-DX=1") == 0
    tree.age()
    tree.touch("a.cu")
    assert tree.library() == 3                                     # b as well: it was made with the define
    tree.monkeypatch.setenv("NVCC", str(tree.d / "other_nvcc"))
    assert tree.library() == 3 and tree.library() == 0


def test_a_build_that_failed_is_tried_again(tree):
    assert tree.library() == 3
    tree.monkeypatch.setattr(build, "UNITS", ["a.cu", "fail.cu"])
    (tree.d / "fail.cu").write_text("")
    for _ in range(2):
        with pytest.raises(RuntimeError):
            tree.library()
    assert len((tree.d / "calls").read_text().splitlines()) == 1   # a.cu stands
    tree.monkeypatch.setattr(build, "UNITS", ["a.cu"])
    assert tree.library() == 1 and tree.library() == 0


def test_the_binding_is_made_again_for_another_torch_or_python(tree):
    assert tree.marshal() == 1 and tree.marshal() == 0
    tree.age()
    tree.touch("serving_marshal.cpp")
    assert tree.marshal() == 1 and tree.marshal() == 0
    tree.monkeypatch.setattr(torch, "__version__", "0.0")
    assert tree.marshal() == 1 and tree.marshal() == 0
    tree.monkeypatch.setattr(sys, "version", "3.99.0 (of a test)")
    assert tree.marshal() == 1 and tree.marshal() == 0
    tree.monkeypatch.setenv("CXX", str(tree.d / "nvcc"))
    assert tree.marshal() == 1
