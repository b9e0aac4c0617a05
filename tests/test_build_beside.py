"""The native half of the binding is compiled beside the library's sources, not before or behind them."""
import os
import subprocess
import threading

import pytest

from paper_2604_16498_b200 import build


def _tree(monkeypatch, tmp_path, sources):
    for name, path in (("HERE", ""), ("CSRC", "csrc"), ("INCLUDE", "include"), ("LIB", "libforge.so"), ("HOST_CALLS", "host_calls.x.so"), ("OBJ_DIR", "obj")):
        monkeypatch.setattr(build, name, str(tmp_path / path))
    for name in (*(f"csrc/{s}.cu" for s in sources), "csrc/host_calls.cpp", "include/forge.h"):
        (tmp_path / name).parent.mkdir(exist_ok=True)
        (tmp_path / name).write_text("")


def _write(cmd):
    with open(cmd[cmd.index("-o") + 1], "w") as f:
        f.write(" ".join(cmd))


@pytest.mark.parametrize("sources", ["ab", "abcdefghij"])
def test_the_module_is_built_beside_the_library(monkeypatch, tmp_path, sources):
    """g++ ends only when a source is being compiled, and that source's compiler only when g++ is running."""
    _tree(monkeypatch, tmp_path, sources)
    gxx, nvcc, ran = threading.Event(), threading.Event(), []

    def run(cmd, **kw):
        name = os.path.basename(cmd[0])
        mine, other = (gxx, nvcc) if name == "g++" else (nvcc, gxx)
        mine.set()
        met = "-shared" in cmd and name == "nvcc" or other.wait(20)
        ran.append((name, "-shared" in cmd))
        _write(cmd)
        return subprocess.CompletedProcess(cmd, 0 if met else 1, "", "nobody there")
    monkeypatch.setattr(build.subprocess, "run", run)
    assert build.build() == str(tmp_path / "libforge.so")
    assert (tmp_path / "libforge.so").exists() and (tmp_path / "host_calls.x.so").exists()
    assert sorted(ran) == sorted([("g++", True)] + [("nvcc", False)] * len(sources) + [("nvcc", True)])
    assert ran[-1] == ("nvcc", True)  # the link behind all


@pytest.mark.parametrize("broken", ["g++", "nvcc"])
def test_one_that_fails_does_not_take_the_other_along(monkeypatch, tmp_path, broken, capsys):
    _tree(monkeypatch, tmp_path, "abc")

    def run(cmd, **kw):
        bad = os.path.basename(cmd[0]) == broken
        if not bad:
            _write(cmd)
        return subprocess.CompletedProcess(cmd, int(bad), "", "it does not compile")
    monkeypatch.setattr(build.subprocess, "run", run)
    if broken == "nvcc":
        with pytest.raises(RuntimeError, match="nvcc failed"):
            build.build()
        assert (tmp_path / "host_calls.x.so").exists() and not (tmp_path / "libforge.so").exists()
    else:
        build.build()
        assert (tmp_path / "libforge.so").exists() and not (tmp_path / "host_calls.x.so").exists()
        assert "it does not compile" in capsys.readouterr().err
