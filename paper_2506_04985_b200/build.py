"""Builds the C-ABI shared library in-tree with nvcc for sm_100a, and the extension that marshals its attention calls.

    python -m paper_2506_04985_b200.build [-v]

The library is a plain `nvcc -shared` of csrc/*.cu (no torch headers), the extension a `g++ -shared` of csrc/calls.cpp
against torch's headers and libraries; each is rebuilt when a source is newer than the binary, the extension also when it was
built for another torch or interpreter.
"""
import glob
import importlib.util
import os
import subprocess
import sys

HERE = os.path.dirname(os.path.abspath(__file__))
LIB = os.path.join(HERE, "libfpt_b200.so")
SRC = sorted(glob.glob(os.path.join(HERE, "csrc", "*.cu")))
DEPS = SRC + sorted(glob.glob(os.path.join(HERE, "csrc", "*.cuh")) + glob.glob(os.path.join(HERE, "csrc", "*.h"))) + [
    os.path.join(os.path.dirname(HERE), "include", "fpt.h")]


CALLS = os.path.join(HERE, "_calls.so")
CALLS_SRC = os.path.join(HERE, "csrc", "calls.cpp")


def nvcc_path():
    for cand in (os.environ.get("NVCC"), "/usr/local/cuda/bin/nvcc", "nvcc"):
        if cand and (os.path.isabs(cand) and os.path.exists(cand) or not os.path.isabs(cand)):
            return cand
    return "nvcc"


def _older(binary, sources):
    if not os.path.exists(binary):
        return True
    t = os.path.getmtime(binary)
    return any(os.path.getmtime(f) > t for f in sources)


def needs_build():
    return _older(LIB, DEPS)


def _run(cmd, what, verbose):
    r = subprocess.run(cmd, stdout=subprocess.PIPE, stderr=subprocess.STDOUT, text=True)
    if verbose or r.returncode != 0:
        sys.stderr.write(r.stdout)
    if r.returncode != 0:
        raise RuntimeError(f"{os.path.basename(cmd[0])} failed building " + what)


def calls_abi():
    """What the extension is bound to: the interpreter's and torch's versions, which it carries as a text."""
    import torch
    return f"python {sys.version_info[0]}.{sys.version_info[1]} torch {torch.__version__}"


def _calls_fit():
    if _older(CALLS, [CALLS_SRC, DEPS[-1]]):
        return False
    with open(CALLS, "rb") as f:
        return calls_abi().encode() + b"\0" in f.read()


def build_calls(verbose=False, force=False):
    if not force and _calls_fit():
        return CALLS
    import sysconfig
    import torch
    top = os.path.dirname(torch.__file__)
    inc = [os.path.join(top, "include"), os.path.join(top, "include", "torch", "csrc", "api", "include"),
           sysconfig.get_paths()["include"], os.path.join(os.path.dirname(os.path.dirname(os.path.realpath(nvcc_path()))), "include")]
    cmd = ([os.environ.get("CXX", "g++"), "-O2", "-std=c++17", "-fPIC", "-shared", f'-DFPT_CALLS_ABI="{calls_abi()}"'] +
           [f for i in inc for f in ("-isystem", i)] + [CALLS_SRC, "-o", CALLS, "-L" + os.path.join(top, "lib"), "-lc10", "-lc10_cuda", "-ltorch_cpu", "-ltorch_python"])
    _run(cmd, CALLS, verbose)
    return CALLS


def build(verbose=False, force=False):
    if force or needs_build():
        cmd = [nvcc_path(), "-gencode", "arch=compute_100a,code=sm_100a", "-lineinfo", "-O3", "-std=c++17",
               "-Xcompiler", "-fPIC", "-shared", "-o", LIB] + SRC
        if verbose:
            cmd += ["-Xptxas", "-v"]
        _run(cmd, LIB, verbose)
    if importlib.util.find_spec("torch"):        # without torch there is nobody to marshal for: the C library alone
        build_calls(verbose, force)
    return LIB


if __name__ == "__main__":
    print(build(verbose="-v" in sys.argv, force=True))
