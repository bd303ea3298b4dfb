"""How the attention calls deal out their work (csrc/attn_rules.h), compiled for the host."""
import ctypes
import functools
import os
import subprocess
import tempfile

CSRC = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2506_04985_b200", "csrc")

SOURCE = """
#include "attn_rules.h"
using namespace fpt;
extern "C" int fits(int lo, int hi, int M) { return rows_fit(lo, hi, M); }
extern "C" int place(int lo, int hi, int s, int block, int id) { return place_of_task(lo, hi, s, block, id); }
extern "C" long long tasks(int M, int n_seqs, int block) { return block_tasks(M, n_seqs, block); }
"""


@functools.lru_cache(None)
def rules():
    with tempfile.TemporaryDirectory() as tmp:
        src, lib = os.path.join(tmp, "rules.cpp"), os.path.join(tmp, "librules.so")
        with open(src, "w") as f:
            f.write(SOURCE)
        subprocess.run(["g++", "-std=c++17", "-O1", "-Wall", "-Werror", "-shared", "-fPIC", "-I", CSRC, src, "-o", lib], check=True)
        L = ctypes.CDLL(lib)
        L.tasks.restype = ctypes.c_longlong
        return L
