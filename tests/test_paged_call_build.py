"""The extension module of the paged operators' calls: built for one torch, and by several processes at once (no GPU)."""
import os
import subprocess
import sys

import pytest
import torch

from paper_2503_08524_b200 import build

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


@pytest.fixture
def compiler(monkeypatch, tmp_path):
    """A g++ that writes its command line's sources into the output, in a package folder of its own; calls are kept."""
    calls = []
    (tmp_path / "csrc").mkdir()
    (tmp_path / "csrc" / "paged_call.cpp").write_text("//")
    monkeypatch.setattr(build, "PKG", str(tmp_path))
    monkeypatch.setattr(build, "CSRC", str(tmp_path / "csrc"))
    monkeypatch.setattr(build, "CALL", str(tmp_path / "_paged_call.so"), raising=False)

    def run(cmd, **kw):
        out = cmd[cmd.index("-o") + 1]
        calls.append(out)
        with open(out, "w") as f:
            f.write("half")
            f.flush()
            nested = getattr(run, "meanwhile", None)
            if nested:                       # another process gets as far in the middle of this one
                run.meanwhile = None
                nested()
            f.write(" and half")
        return subprocess.CompletedProcess(cmd, run.status, "", "")

    run.status = 0
    monkeypatch.setattr(build.subprocess, "run", run)
    run.calls = calls
    return run


def test_a_module_built_for_another_torch_is_not_taken(compiler, monkeypatch):
    first = build.build_call()
    assert build.build_call() == first and len(compiler.calls) == 1      # up to date
    monkeypatch.setattr(torch, "__version__", "9.9.9+other")
    second = build.build_call()
    assert len(compiler.calls) == 2 and second != first
    monkeypatch.setattr(torch._C, "_GLIBCXX_USE_CXX11_ABI", not torch._C._GLIBCXX_USE_CXX11_ABI)
    assert build.build_call() not in (first, second) and len(compiler.calls) == 3


def test_builds_side_by_side_leave_a_whole_module(compiler):
    done = []
    compiler.meanwhile = lambda: done.append(build.build_call())
    out = build.build_call()
    assert done == [out] and len(set(compiler.calls)) == 2               # no file is written by two
    assert open(out).read() == "half and half"
    assert sorted(n for n in os.listdir(build.PKG) if n.startswith("_paged_call")) == [os.path.basename(out)]


def test_a_build_that_fails_leaves_nothing(compiler):
    compiler.status = 1
    with pytest.raises(RuntimeError, match="g\\+\\+ failed"):
        build.build_call()
    assert not [n for n in os.listdir(build.PKG) if n.startswith("_paged_call")]


def test_processes_that_import_at_once():
    out = build.build_call()
    os.utime(out, (1, 1))                    # stale for all of them
    code = "from paper_2503_08524_b200 import paged; print(paged._paged_call.__file__)"
    ps = [subprocess.Popen([sys.executable, "-c", code], cwd=ROOT, stdout=subprocess.PIPE, stderr=subprocess.PIPE, text=True) for _ in range(3)]
    for p in ps:
        got, err = p.communicate(timeout=600)
        assert p.returncode == 0 and got.strip() == out, err[-2000:]
