"""How the attention calls deal out their work (csrc/attn_rules.h), compiled for the host."""
import collections
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
extern "C" int range_first(int each, int longer, int i) { return Ranges{each, longer}.first_of(i); }
extern "C" int range_of(int each, int longer, int x) { return Ranges{each, longer}.cta_of(x); }
extern "C" int dec_tiles(int len) { return tiles_of(len); }
extern "C" int part_limits(int which) { return which == 0 ? kPrTile : which == 1 ? kPrPartTiles : kPrParts; }
extern "C" int first_length(unsigned all, int sms) { return Splitting::first_length(all, sms); }
extern "C" void splitting(int len_k, int len_q, int places, int per_log2, int causal, int L, long long* out) {
  const Splitting s = {len_k, len_q, places, per_log2, causal};
  out[0] = s.most(); out[1] = s.tiles(); out[2] = s.split(L); out[3] = s.parts(L);
}
"""


Split = collections.namedtuple("Split", "most tiles split parts")


def splitting(len_k, len_q, per_log2, causal, L):
    """How the tasks (of 2^per_log2 rows) of a sequence are split where a part has at most L tiles of keys."""
    out = (ctypes.c_longlong * 4)()
    rules().splitting(len_k, len_q, -(-len_q // (1 << per_log2)), per_log2, int(causal), L, out)
    return Split(*out)


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
