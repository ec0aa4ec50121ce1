"""The build's choice of what to compile, without compiling."""
import sys

import pytest

from paper_2008_05823_b200 import build


def run(monkeypatch, tmp_path, torch_there):
    """The commands of a forced build into an empty folder."""
    commands = []
    monkeypatch.setattr(build, "HERE", str(tmp_path))
    monkeypatch.setattr(build.subprocess, "check_call", lambda cmd, **kw: commands.append(cmd))
    if not torch_there:
        monkeypatch.setitem(sys.modules, "torch", None)               # import torch raises ImportError
        monkeypatch.setitem(sys.modules, "torch.utils", None)
    return build.build(force=True), commands


def test_everything_is_built(monkeypatch, tmp_path):
    pytest.importorskip("torch")
    outs, commands = run(monkeypatch, tmp_path, True)
    assert len(outs) == len(commands) == len(build.TARGETS)


def test_the_libraries_are_built_without_torch(monkeypatch, tmp_path, capsys):
    """The C library and the generator need nvcc alone; what is C++ against torch is left out with a word."""
    outs, commands = run(monkeypatch, tmp_path, False)
    built = [name for name in build.TARGETS if name != "_host.so"]
    assert [o.rsplit("/", 1)[1] for o in outs] == built and len(commands) == len(built)
    assert "_host.so" in capsys.readouterr().err
