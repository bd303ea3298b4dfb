"""How the attention calls deal out their work: the compiled rules of csrc/attn_rules.h, without a GPU."""
import os
import re

import numpy as np

from attn_rules import CSRC, rules


def packed(rng, n, longest, before, behind):
    lens = rng.integers(0, longest, n)
    cu = np.concatenate([[int(rng.integers(0, before))], lens]).cumsum().tolist()
    return [int(c) for c in cu], int(cu[-1] + rng.integers(0, behind))


def test_every_page_that_packed_rows_touch_has_one_task():
    """The pages (at any offset of the first row in its page) that a sequence touches have a place each among its tasks, and a task belongs
    to one sequence."""
    R, rng = rules(), np.random.default_rng(1)
    for _ in range(60):
        n, block = int(rng.integers(1, 50)), int(rng.choice([0, 16, 32, 64, 128]))
        cu, M = packed(rng, n, 200, 50, 40)
        total = R.tasks(M, n, block)
        seen = [set() for _ in range(n)]
        for task in range(total):
            own = [(s, R.place(cu[s], cu[s + 1], s, block, task)) for s in range(n)]
            own = [(s, p) for s, p in own if p >= 0]
            assert len(own) <= 1
            for s, p in own:
                seen[s].add(p if block else task - cu[s])
        for s in range(n):
            length = cu[s + 1] - cu[s]
            need = length if block == 0 else 0 if length == 0 else (block - 1 + length - 1) // block + 1
            assert set(range(need)) <= seen[s], (cu, s, block)


def test_offsets_that_do_not_ascend_are_refused_or_share_tasks():
    """Two sequences that are fine by themselves can both have a task where one between them is not: why a task has to be
    given to one of them as a whole."""
    R = rules()
    cu, M, block = [0, 1000, 5, 1000], 1000, 64
    assert [R.fits(cu[s], cu[s + 1], M) for s in range(3)] == [1, 0, 1]
    both = [t for t in range(R.tasks(M, 3, block)) if all(R.place(cu[s], cu[s + 1], s, block, t) >= 0 for s in (0, 2))]
    assert both
    for lo, hi in ((-1, 5), (5, 4), (0, 1001), (2 ** 31 - 1, 2 ** 31 - 1), (-2 ** 31, -2 ** 31)):
        assert not R.fits(lo, hi, M)


def test_one_thread_says_what_was_found():
    """Several threads may claim a task (offsets that do not ascend).  Only the one whose claim is the first stores what it found: five words
    stored by two threads could mix a first row with another's rows; and it is a task only where there was no second."""
    text = open(os.path.join(CSRC, "attn_common.cuh")).read()
    body = text[text.index("bool find_task("):]
    body = body[:body.index("\n}\n")]
    assert re.findall(r"[^;{}\n]*\*found\s*=", body) == ["      if (place >= 0 && atomicAdd(&claims, 1) == 0) *found ="]
    assert "found->" not in body and re.search(r"claims = 0;\s*__syncthreads\(\);", body) and body.rstrip().endswith("__syncthreads();\n  return claims == 1;")
