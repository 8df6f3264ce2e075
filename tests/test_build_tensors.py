"""The module that checks tensors for the bindings is optional: the library is built without it."""
import os
import subprocess

import pytest

from paper_2603_06274_amd import build


@pytest.fixture
def elsewhere(tmp_path, monkeypatch):
    """A build that compiles nothing, into a folder of its own."""
    made = []
    monkeypatch.setattr(build, "LIB", str(tmp_path / "lib.so"))
    monkeypatch.setattr(build, "OBJ", str(tmp_path))
    monkeypatch.setattr(build, "TENSORS", str(tmp_path / os.path.basename(build.TENSORS)))
    monkeypatch.setattr(build, "check_wait_states", lambda extra=(): made.append("wait states"))
    monkeypatch.setattr(build, "_compile", lambda src, extra: made.append(src) or src)
    monkeypatch.setattr(build.subprocess, "run", lambda cmd, **kw: made.append("link") or subprocess.CompletedProcess(cmd, 0, "", ""))
    return made


@pytest.mark.parametrize("why", [ModuleNotFoundError("No module named 'torch'"), RuntimeError("Python.h: No such file or directory")])
def test_the_library_is_built_without_it(elsewhere, monkeypatch, capsys, why):
    def fails():
        raise why

    monkeypatch.setattr(build, "build_tensors", fails)
    open(build.TENSORS, "w").close()               # one of an earlier build, of which nobody knows whether it still fits
    assert build.build(verbose=False) == build.LIB
    assert elsewhere[-1] == "link" and "wait states" in elsewhere
    assert str(why) in capsys.readouterr().err and not os.path.exists(build.TENSORS)
