"""What build_library does where only hipcc is there: the library is built, and the compiled part of the binding, which needs g++ and the headers of torch
and Python, is left out and none of an earlier build stays behind (no GPU needed; no compiler is run)."""
import os
import shutil
import subprocess
import sys
import sysconfig

import pytest

from paper_2404_14469_amd import build


@pytest.fixture
def commands(monkeypatch, tmp_path):
    """The commands that would have run; those of g++ fail."""
    ran = []

    class Done:
        returncode = 0

        def __init__(self, cmd, **_):
            ran.append(cmd[0])

        def communicate(self):
            return b"", None

    def call(cmd, **_):
        ran.append(cmd[0])
        if cmd[0] == "g++":
            raise subprocess.CalledProcessError(1, cmd)
    monkeypatch.setattr(build.subprocess, "Popen", Done)
    monkeypatch.setattr(build.subprocess, "check_call", call)
    monkeypatch.setattr(build, "STEPS", str(tmp_path / "_steps.so"))
    (tmp_path / "_steps.so").write_text("of an earlier build")
    return ran


@pytest.mark.parametrize("missing", ["compiler", "torch", "torch's headers", "Python's headers"])
def test_library_alone(commands, monkeypatch, missing, capsys):
    if missing == "compiler":
        monkeypatch.setattr(shutil, "which", lambda name, *a, **k: None)
    elif missing == "torch":
        monkeypatch.setitem(sys.modules, "torch", None)
    elif missing == "torch's headers":
        from torch.utils import cpp_extension
        monkeypatch.setattr(cpp_extension, "include_paths", lambda *a, **k: ["/nonexistent"])
    else:
        monkeypatch.setattr(sysconfig, "get_paths", lambda *a, **k: {"include": "/nonexistent"})
    assert build.build_library() == build.LIB
    assert commands == [build.HIPCC] * (len(build.SOURCES) + 1)
    assert not os.path.exists(build.STEPS)
    assert "_steps.so" in capsys.readouterr().out


def test_a_failed_compilation_is_an_error(commands):
    with pytest.raises(subprocess.CalledProcessError):
        build.build_library()
    assert not os.path.exists(build.STEPS)
