"""Building the library and the binding's native part: without torch, and by several who need it at once. The compilers are stood in
for by what writes files (no device)."""
import importlib.machinery
import importlib.util
import os
import subprocess
import sys
import time

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


COMPILER = """#!{python}
import os, sys, time
to = sys.argv[sys.argv.index("-o") + 1]
with open({log!r}, "a") as f:
    f.write(to + "\\n")
with open(to, "wb", buffering=0) as f:
    f.write(b"x" * 1000)
    time.sleep(1.0)
    f.write(b"y" * 1000)
"""

FIRST_USE = """
import sys, threading
sys.path.insert(0, {root!r})
from paper_2502_01681_amd import build
build.HERE = {here!r}
build.OBJ = {here!r} + "/_build"
build.LIB = {here!r} + "/libdg4.so"
build.SOURCES = build.SOURCES[:1]
print("ready", flush=True)
sys.stdin.readline()
got = []
def run():
    path = build.{what}()
    got.append(open(path, "rb").read() == b"x" * 1000 + b"y" * 1000)
threads = [threading.Thread(target=run) for _ in range(3)]
[t.start() for t in threads]
[t.join() for t in threads]
assert got == [True] * 3, got
"""


@pytest.mark.parametrize("what", ["marshal", "library"])
def test_those_who_need_it_first_wait_for_one_build(tmp_path, what):
    """Three threads in each of three processes, started while a slow compiler has written half of it: one build, and every one of
    them reads it whole."""
    log, compiler = tmp_path / "log", tmp_path / "compiler"
    compiler.write_text(COMPILER.format(python=sys.executable, log=str(log)))
    compiler.chmod(0o755)
    env = dict(os.environ, CXX=str(compiler), HIPCC=str(compiler))
    code = FIRST_USE.format(root=build.ROOT, here=str(tmp_path), what=what)
    users = [subprocess.Popen([sys.executable, "-c", code], env=env, stdin=subprocess.PIPE, stdout=subprocess.PIPE, text=True) for _ in range(3)]
    for u in users:
        assert u.stdout.readline() == "ready\n"
    for u in users:
        u.stdin.write("go\n")
        u.stdin.flush()
        time.sleep(0.3)
    for u in users:
        u.communicate(timeout=60)
        assert u.returncode == 0
    written = [os.path.basename(x) for x in log.read_text().split()]
    assert sorted(set(written)) == sorted(written), written


def test_a_module_of_other_sources_or_another_torch_is_not_taken(tmp_path, monkeypatch):
    here = build._marshal_path()
    assert here == build._marshal_path() and here.endswith(importlib.machinery.EXTENSION_SUFFIXES[0])
    header = tmp_path / "dg4_mx4.h"
    header.write_text("other")
    with monkeypatch.context() as m:
        m.setattr(build, "MARSHAL_HEADERS", build.MARSHAL_HEADERS[:-1] + [str(header)])
        assert build._marshal_path() != here
    (tmp_path / "version.py").write_text("__version__ = '0'")
    with monkeypatch.context() as m:
        m.setattr(build, "_torch", lambda: str(tmp_path))
        assert build._marshal_path() != here


def test_a_build_leaves_the_module_that_it_is_for(elsewhere):
    old = os.path.join(build.HERE, "_dg4_marshal-of-old.so")
    open(old, "w").close()
    build.build()
    assert os.listdir(build.HERE).count(os.path.basename(old)) == 0 and os.path.exists(build._marshal_path()) and len(modules(elsewhere)) == 1
    build.build(force=False)
    assert len(modules(elsewhere)) == 1
