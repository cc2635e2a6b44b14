"""The build's decisions without a compiler: what is made anew, and what a failing part leaves behind."""
import os
import subprocess

import pytest
import torch

from paper_2607_10661_gb300 import _build, ptd


class Tree:
    """A package of its own with two kernels' sources, and compilers that write a file."""

    def __init__(self, tmp_path, monkeypatch):
        self.ran, self.failing = [], ()
        pkg = tmp_path / "pkg"
        csrc = pkg / "csrc"
        csrc.mkdir(parents=True)
        (tmp_path / "include").mkdir()
        for f in (csrc / "a.cu", csrc / "b.cu", csrc / "pycall.cpp", tmp_path / "include" / "ptd.h"):
            f.write_text("")
            os.utime(f, (1e9, 1e9))
        old = _build.PKG
        for name, value in list(vars(_build).items()):   # every path of the package
            if isinstance(value, str) and value.startswith(old):
                monkeypatch.setattr(_build, name, str(pkg) + value[len(old):])
        monkeypatch.setattr(_build, "nvcc", lambda: "nvcc")
        monkeypatch.setattr(subprocess, "run", self.run)

    def run(self, cmd, **kw):
        out = os.path.basename(cmd[cmd.index("-o") + 1])
        self.ran.append(out)
        failed = out in self.failing
        if not failed:
            open(cmd[cmd.index("-o") + 1], "w").close()
        return subprocess.CompletedProcess(cmd, int(failed), "", "no such header" if failed else "")

    def build(self, **kw):
        del self.ran[:]
        _build.build(**kw)
        return sorted(self.ran)


ALL = ["_ptdcall.so.tmp", "a.o", "b.o", "libptd.so.tmp"]


@pytest.fixture
def tree(tmp_path, monkeypatch):
    return Tree(tmp_path, monkeypatch)


def test_call_module_is_made_anew_for_another_torch(tree, monkeypatch):
    assert tree.build() == ALL and tree.build() == [] and tree.build(force=True) == ALL
    monkeypatch.setattr(torch, "__version__", torch.__version__ + ".other")
    assert tree.build() == ["_ptdcall.so.tmp"] and tree.build() == []


def test_call_module_is_made_anew_where_nothing_says_what_it_is_for(tree):
    tree.build()
    os.remove(_build.CALLS_FOR)
    assert tree.build() == ["_ptdcall.so.tmp"] and tree.build() == []


def test_library_is_linked_where_the_call_module_does_not_compile(tree):
    tree.failing = ("_ptdcall.so.tmp",)
    with pytest.raises(RuntimeError, match=r"pycall.cpp[^$]*no such header"):
        tree.build()
    assert sorted(tree.ran) == ALL and os.path.exists(_build.LIB) and not os.path.exists(_build.CALLS)
    tree.failing = ()
    tree.build()
    assert os.path.exists(_build.CALLS) and tree.build() == []


def test_call_module_of_another_torch_is_refused(monkeypatch):
    import __graft_entry__

    __graft_entry__.build()
    ptd._native()
    monkeypatch.setattr(ptd, "_calls", None)
    monkeypatch.setattr(torch, "__version__", torch.__version__ + ".other")
    try:
        with pytest.raises(RuntimeError, match="compiled for torch .*, this is .*other"):
            ptd._native()
    finally:
        monkeypatch.undo()
        ptd._calls = None
        ptd._native()
