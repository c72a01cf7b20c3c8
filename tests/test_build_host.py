"""libhf.so is built without torch; the host library belongs to the torch that it was built against.  The commands are recorded, none is run."""
import os
import sys

import pytest

from paper_2604_10103_b200 import binding, build


@pytest.fixture
def commands(monkeypatch):
    ran = []
    monkeypatch.setattr(build, "_run", lambda cmd: ran.append(cmd) or "")
    return ran


def outputs(commands):
    return [os.path.basename(c[c.index("-o") + 1]) for c in commands]


def test_without_torch(commands, monkeypatch, capsys):
    monkeypatch.setitem(sys.modules, "torch", None)
    assert build.build(force=True) == build.LIB and outputs(commands) == ["libhf.so"]
    assert "torch is not installed" in capsys.readouterr().err
    monkeypatch.setattr(build, "_older", lambda lib, deps: lib != build.LIB)
    assert not build.stale()


def test_a_host_library_that_fails_leaves_the_other_built(monkeypatch):
    ran = []

    def run(cmd):
        ran.append(cmd)
        if build.HOST_SOURCE in cmd:
            raise RuntimeError("g++ failed: Python.h is missing")
        return ""
    monkeypatch.setattr(build, "_run", run)
    with pytest.raises(RuntimeError, match="Python.h"):
        build.build(force=True)
    assert outputs(ran)[0] == "libhf.so" and len(ran) == 2


def test_another_torch_has_a_library_of_its_own(commands, monkeypatch):
    import torch
    build.build(force=True)
    mine = outputs(commands)
    assert mine == ["libhf.so", f"libhf_host-{torch.__version__}.so"] and os.path.basename(build.host_lib()) == mine[1]
    monkeypatch.setattr(torch, "__version__", "2.99.0+test")
    monkeypatch.setattr(build, "_older", lambda lib, deps: os.path.basename(lib) not in mine)
    assert build.stale()
    commands.clear()
    build.build()
    assert outputs(commands) == ["libhf_host-2.99.0+test.so"]
    monkeypatch.setattr(binding, "_host", None)
    with pytest.raises(RuntimeError, match="2.99.0.*is missing"):
        binding.host()
