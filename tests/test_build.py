"""Building the library and the binding's native part: without torch, and by several who need it at once. The compilers are stood in
for by what writes files (no device)."""
import importlib.util
import os
import subprocess

import pytest

from paper_2502_01681_amd import build


@pytest.fixture
def elsewhere(tmp_path, monkeypatch):
    """The build's outputs in a folder of the test, its commands recorded: each writes what -o names."""
    for name in ("HERE", "OBJ", "LIB"):
        monkeypatch.setattr(build, name, str(tmp_path / os.path.basename(getattr(build, name))))
    os.makedirs(build.HERE)
    commands = []

    def check_call(command, **kw):
        commands.append(command)
        with open(command[command.index("-o") + 1], "w") as f:
            f.write(" ".join(command))
    monkeypatch.setattr(build.subprocess, "check_call", check_call)
    monkeypatch.delenv("CXX", raising=False)
    monkeypatch.delenv("HIPCC", raising=False)
    return commands


def linked(commands):
    return [c for c in commands if "-shared" in c and "hipcc" in c[0]]


def modules(commands):
    return [c for c in commands if "-ltorch_python" in c]


def test_the_library_needs_no_torch(elsewhere, monkeypatch):
    find = importlib.util.find_spec
    monkeypatch.setattr(importlib.util, "find_spec", lambda name, *a: None if name == "torch" else find(name, *a))
    for force in (True, False):
        assert build.build(force=force) == build.LIB
        assert os.path.exists(build.LIB) and len(linked(elsewhere)) == 1 and not modules(elsewhere)


def test_the_library_does_not_wait_for_a_module_that_cannot_be_built(elsewhere, monkeypatch):
    write = build.subprocess.check_call

    def check_call(command, **kw):
        if "-ltorch_python" in command:
            raise subprocess.CalledProcessError(1, command)
        write(command)
    monkeypatch.setattr(build.subprocess, "check_call", check_call)
    with pytest.raises(subprocess.CalledProcessError):
        build.build()
    assert os.path.exists(build.LIB) and len(linked(elsewhere)) == 1
