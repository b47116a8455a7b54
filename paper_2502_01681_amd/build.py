"""Build libdg4.so (HIP kernels + C ABI) in-tree for gfx950 and, where torch is installed, the native part of the Python binding."""
from __future__ import annotations

import contextlib
import fcntl
import glob
import hashlib
import importlib.machinery
import importlib.util
import os
import subprocess
import sysconfig
from concurrent.futures import ThreadPoolExecutor

HERE = os.path.dirname(os.path.abspath(__file__))
ROOT = os.path.dirname(HERE)
CSRC = os.path.join(HERE, "csrc")
LIB = os.path.join(HERE, "libdg4.so")
OBJ = os.path.join(HERE, "_build")
SOURCES = ["dg4_graph.cpp", "dg4_graph_gpu.hip", "dg4_api.cpp", "dg4_kernels.hip", "dg4_sweep.hip", "dg4_flow.hip", "dg4_heads.hip",
           "dg4_static.hip", "dg4_kv8.hip", "dg4_lora.hip", "dg4_kv4.hip", "dg4_mx4.hip"]
HEADERS = [os.path.join(CSRC, h) for h in ("dg4_internal.h", "dg4_device.h", "dg4_rowops.h", "dg4_wait.h", "dg4_fp4.h")] + [os.path.join(ROOT, "include", h) for h in ("dg4.h", "dg4_serving.h", "dg4_mx4.h")]

MARSHAL_SOURCE = os.path.join(CSRC, "dg4_marshal.cpp")
MARSHAL_HEADERS = [os.path.join(ROOT, "include", h) for h in ("dg4.h", "dg4_serving.h", "dg4_mx4.h")]


def sources():
    return [os.path.join(CSRC, s) for s in SOURCES]


def _torch():
    """Folder of torch, None without it (which is not imported)."""
    spec = importlib.util.find_spec("torch")
    return spec and os.path.dirname(spec.origin)


def _older(path, sources) -> bool:
    return not os.path.exists(path) or any(os.path.getmtime(d) > os.path.getmtime(path) for d in sources)


def _marshal_path() -> str:
    """Where the native part of the binding stands: by the interpreter, torch and sources that it is built from, so that a module of
    others is not taken for it."""
    digest = hashlib.sha256()
    for path in [os.path.join(_torch(), "version.py"), MARSHAL_SOURCE] + MARSHAL_HEADERS:
        with open(path, "rb") as f:
            digest.update(f.read())
    # (the suffix not from sysconfig, whose first use is not for two threads at once)
    return os.path.join(HERE, "_dg4_marshal-" + digest.hexdigest()[:12] + importlib.machinery.EXTENSION_SUFFIXES[0])


def stale() -> bool:
    return _older(LIB, sources() + HEADERS) or _torch() is not None and not os.path.exists(_marshal_path())


@contextlib.contextmanager
def _alone():
    """One at a time builds, among threads and processes."""
    os.makedirs(OBJ, exist_ok=True)
    with open(os.path.join(OBJ, "lock"), "w") as f:
        fcntl.flock(f, fcntl.LOCK_EX)
        yield


def _write(path, command):
    """command, a link of which -o is `path`: what stands there is whole at any time, and mapped files are not written to."""
    new = os.path.join(OBJ, os.path.basename(path))
    subprocess.check_call(command + ["-o", new])
    os.replace(new, path)


def _flags():
    return ["-O3", "-std=c++17", "-fPIC", "--offload-arch=gfx950", "-x", "hip",
            # packed fp32 VALU forms are switched off for every kernel of this library
            "-Xclang", "-target-feature", "-Xclang", "-packed-fp32-ops",
            # MFMA accumulators in VGPRs: leaves the AGPR half of the register file to the
            # weights that the persistent sweep kernel keeps resident
            "-mllvm", "-amdgpu-mfma-vgpr-form=1",
            # no wave-wide rewriting of atomics: the ticket draws of the persistent kernels are single-lane
            # already, and the rewriting makes the wave wait for the result on the spot
            "-mllvm", "-amdgpu-atomic-optimizer-strategy=None",
            "-I", os.path.join(ROOT, "include"), "-I", CSRC,
            "-Wall", "-Wno-unused-function"]


def _build_marshal(path):
    """The native part of the Python binding (host code, against this interpreter and torch)."""
    torch = _torch()
    _write(path, [os.environ.get("CXX", "g++"), "-O2", "-std=c++17", "-fPIC", "-shared", "-Wall", "-I", sysconfig.get_paths()["include"],
                  "-isystem", os.path.join(torch, "include"), "-I", os.path.join(ROOT, "include"), MARSHAL_SOURCE,
                  "-L", os.path.join(torch, "lib"), "-ltorch_python", "-ltorch_cpu", "-lc10"])


def library() -> str:
    """Path of the shared library, built first if it is not there."""
    if not os.path.exists(LIB):
        with _alone():
            if not os.path.exists(LIB):
                _build(force=True)
    return LIB


def marshal() -> str:
    """Path of the native part of the binding, built first if it is not there."""
    path = _marshal_path()
    if not os.path.exists(path):
        with _alone():
            if not os.path.exists(path):
                _build_marshal(path)
    return path


def build(force: bool = True) -> str:
    """Compile every source with hipcc for gfx950 (one object per source, in parallel) and link the
    shared library, whether or not the module beside it can be built. force=False recompiles only the sources
    that changed since their object was made."""
    with _alone():
        return LIB if not force and not stale() else _build(force)


def _build(force):
    hipcc = os.environ.get("HIPCC", "/opt/rocm/bin/hipcc")
    newest_header = max(os.path.getmtime(h) for h in HEADERS)

    def compile_one(src):
        obj = os.path.join(OBJ, os.path.basename(src) + ".o")
        if not force and os.path.exists(obj) and os.path.getmtime(obj) > max(os.path.getmtime(src), newest_header):
            return obj
        subprocess.check_call([hipcc] + _flags() + ["-c", src, "-o", obj], stderr=subprocess.DEVNULL if os.environ.get("DG4_QUIET") else None)
        return obj

    with ThreadPoolExecutor(max_workers=min(8, len(SOURCES))) as ex:
        path = _marshal_path() if _torch() else None
        module = ex.submit(_build_marshal, path) if path and (force or not os.path.exists(path)) else None
        objs = list(ex.map(compile_one, sources()))
        _write(LIB, [hipcc, "-shared", "-fPIC", "--offload-arch=gfx950"] + objs)
        if module is not None:
            module.result()
            for other in glob.glob(os.path.join(HERE, "_dg4_marshal*.so")):    # of sources or a torch that are no more
                if other != path:
                    os.remove(other)
    return LIB


if __name__ == "__main__":
    import sys
    print(build(force="--incremental" not in sys.argv))
