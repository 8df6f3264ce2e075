"""The module that checks tensors for the bindings is optional: the library is built without it."""
import importlib.util
import os
import subprocess
import sys
import sysconfig

import pytest
import torch

from paper_2603_06274_amd import build
from paper_2603_06274_amd import decode_binding as db


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


def test_a_module_that_is_built_is_used():
    """Under a name that other Pythons do not look for.  (What cannot be imported is slower, and would go unnoticed.)"""
    assert build.TENSORS.endswith(sysconfig.get_config_var("EXT_SUFFIX"))
    if not os.path.exists(build.TENSORS):
        pytest.skip("not built")
    assert db._tensors is not None and os.path.samefile(db._tensors.__file__, build.TENSORS)


def test_another_torchs_module_is_refused(tmp_path, monkeypatch):
    path = str(tmp_path / os.path.basename(build.TENSORS))
    monkeypatch.setattr(build, "TENSORS", path)
    try:
        build.build_tensors("2.0.0 " + "0" * 40)
    except (ImportError, RuntimeError):
        pytest.skip("no compiler or headers for it")
    spec = importlib.util.spec_from_file_location("_tensors", path)
    with pytest.raises(ImportError, match="2.0.0 0.*" + torch.version.git_version):
        importlib.util.module_from_spec(spec)


def test_a_module_that_cannot_be_used_says_so(monkeypatch):
    class Finder:
        @staticmethod
        def find_spec(name, path=None, target=None):
            if name.endswith("._tensors"):
                raise ImportError("made for another torch")

    monkeypatch.setattr(sys, "meta_path", [Finder, *sys.meta_path])
    monkeypatch.delitem(sys.modules, "paper_2603_06274_amd._tensors", raising=False)
    spec = importlib.util.spec_from_file_location("paper_2603_06274_amd._checks_in_python", db.__file__)
    plain = importlib.util.module_from_spec(spec)
    with pytest.warns(RuntimeWarning, match="made for another torch"):
        spec.loader.exec_module(plain)
    assert plain._tensors is None and plain._whole(torch.zeros(3, dtype=torch.int32), 3, "x", -1)
