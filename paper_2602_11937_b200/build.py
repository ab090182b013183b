"""In-tree build: the CUDA library (nvcc for sm_100a, one shared object, no torch involved) and the small Python module
through which the binding calls its hot entry points (g++, torch's headers).

``python -m paper_2602_11937_b200.build`` rebuilds when a source is newer than the library made from it.
"""
from __future__ import annotations

import glob
import importlib.util
import os
import platform
import subprocess
import sys
import sysconfig

HERE = os.path.dirname(os.path.abspath(__file__))
CSRC = os.path.join(HERE, "csrc")
LIB_DIR = os.path.join(HERE, "lib")
LIB = os.path.join(LIB_DIR, "libpuzzle_attn.so")
CALL_SRC = os.path.join(CSRC, "call.cpp")
CALL_LIB = os.path.join(LIB_DIR, "_puzzle_call.so")
CALL_STAMP = os.path.join(HERE, "_build", "call.txt")      # what the module was built for
NVCC = os.environ.get("NVCC", "/usr/local/cuda/bin/nvcc")
FLAGS = ["-gencode", "arch=compute_100a,code=sm_100a", "-O3", "-std=c++17", "-lineinfo",
         "-Xcompiler", "-fPIC", "-Xcompiler", "-fvisibility=hidden"]


def sources():
    return sorted(glob.glob(os.path.join(CSRC, "*.cu")))


def _deps():
    return sources() + glob.glob(os.path.join(CSRC, "*.cuh")) + \
        glob.glob(os.path.join(HERE, "..", "include", "*.h")) + [os.path.abspath(__file__)]


def _older(lib: str, deps) -> bool:
    return not os.path.exists(lib) or any(os.path.getmtime(p) > os.path.getmtime(lib) for p in deps)


def is_stale() -> bool:
    return _older(LIB, _deps())


def _torch_dir() -> str:
    return os.path.dirname(importlib.util.find_spec("torch").origin)


def call_target() -> str:
    """The Python and the torch that a build of the native module is good for (their binary interfaces change between
    versions); torch itself is not imported for it."""
    version = {}
    with open(os.path.join(_torch_dir(), "version.py")) as f:
        exec(f.read(), version)
    return "python %s torch %s" % (".".join(platform.python_version_tuple()[:2]), version["__version__"])


def _built_for() -> str:
    try:
        with open(CALL_STAMP) as f:
            return f.read()
    except OSError:
        return ""


def build_call(force: bool = False) -> str:
    """Compile csrc/call.cpp into lib/_puzzle_call.so.  torch has to be imported before it."""
    target = call_target()
    deps = [CALL_SRC, os.path.abspath(__file__)] + glob.glob(os.path.join(HERE, "..", "include", "*.h"))
    if not force and not _older(CALL_LIB, deps) and _built_for() == target:
        return CALL_LIB
    os.makedirs(LIB_DIR, exist_ok=True)
    os.makedirs(os.path.dirname(CALL_STAMP), exist_ok=True)
    torch = _torch_dir()
    include = [os.path.join(torch, "include"), os.path.join(torch, "include", "torch", "csrc", "api", "include"),
               sysconfig.get_paths()["include"], os.path.join(os.path.dirname(os.path.dirname(NVCC)), "include"),
               os.path.join(HERE, "..", "include")]
    tmp = CALL_LIB + ".tmp%d" % os.getpid()
    subprocess.check_call([os.environ.get("CXX", "g++"), "-O2", "-std=c++17", "-fPIC", "-shared", "-fvisibility=hidden", "-w",
                           '-DPUZZLE_BUILT_FOR="%s"' % target,
                           *["-I" + i for i in include], CALL_SRC, "-o", tmp,
                           "-L" + os.path.join(torch, "lib"), "-ltorch_python", "-ltorch_cpu", "-lc10", "-lc10_cuda"])
    os.replace(tmp, CALL_LIB)
    with open(CALL_STAMP, "w") as f:
        f.write(target)
    return CALL_LIB


def build(force: bool = False, verbose: bool = False) -> str:
    """Compile every .cu under csrc/ for sm_100a, link lib/libpuzzle_attn.so, and build the Python module beside it."""
    build_call(force)
    if not force and not is_stale():
        return LIB
    os.makedirs(LIB_DIR, exist_ok=True)
    obj_dir = os.path.join(HERE, "_build")
    os.makedirs(obj_dir, exist_ok=True)
    objs, procs = [], []
    extra = ["-Xptxas", "-v"] if verbose else []
    for src in sources():
        obj = os.path.join(obj_dir, os.path.basename(src)[:-3] + ".o")
        objs.append(obj)
        procs.append((src, subprocess.Popen([NVCC, *FLAGS, *extra, "-c", src, "-o", obj],
                                            stdout=subprocess.PIPE, stderr=subprocess.STDOUT, text=True)))
    for src, p in procs:
        out, _ = p.communicate()
        if verbose or p.returncode != 0:
            sys.stderr.write(out)
        if p.returncode != 0:
            raise RuntimeError("nvcc failed on %s" % src)
    tmp = LIB + ".tmp%d" % os.getpid()
    subprocess.check_call([NVCC, "-shared", "-o", tmp, *objs, "-Xlinker", "--exclude-libs=ALL"])
    os.replace(tmp, LIB)
    return LIB


if __name__ == "__main__":
    print(build(force="--force" in sys.argv, verbose="-v" in sys.argv))
