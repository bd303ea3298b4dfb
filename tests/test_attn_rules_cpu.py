"""How the attention calls deal out their work: the compiled rules of csrc/attn_rules.h, without a GPU."""
import os
import re

import numpy as np

from attn_rules import CSRC, rules, splitting


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


def test_ranges_of_tiles_cover_the_line():
    R, rng = rules(), np.random.default_rng(2)
    for _ in range(100):
        total = int(rng.integers(1, 5000))
        ctas = min(int(rng.integers(1, 500)), total)
        each, longer = total // ctas, total % ctas
        first = [R.range_first(each, longer, i) for i in range(ctas + 1)]
        assert first[0] == 0 and first[-1] == total and min(np.diff(first)) >= 1
        for x in [0, total - 1, *(int(x) for x in rng.integers(0, total, 30))]:
            c = R.range_of(each, longer, x)
            assert first[c] <= x < first[c + 1]
    assert [R.dec_tiles(n) for n in (-5, 0, 1, 64, 65, 2 ** 31 - 257)] == [1, 1, 1, 1, 2, 2 ** 25 - 4]


def tiles_of_places(len_k, len_q, per, causal, tile):
    ends = [min((p + 1) * per, len_q) for p in range(-(-len_q // per))]
    return [-(-(min(max(e + len_k - len_q, 0), len_k) if causal else len_k) // tile) for e in ends]


def test_splitting_takes_the_tasks_with_many_keys():
    """Those, and only those, with more than L tiles, which are the last ones; in parts of at most L, as far as the most parts go."""
    R, rng = rules(), np.random.default_rng(3)
    tile, most_parts = R.part_limits(0), R.part_limits(2)
    for _ in range(3000):
        per_log2, causal = int(rng.integers(4, 9)), bool(rng.integers(0, 2))
        len_q, len_k = (int(np.exp(rng.uniform(0, np.log(top)))) - 1 for top in (5000, 200000))
        L = int(np.exp(rng.uniform(0, np.log(2000))))
        tiles = tiles_of_places(len_k, len_q, 1 << per_log2, causal, tile)
        s = splitting(len_k, len_q, per_log2, causal, L)
        assert s.most == -(-len_k // tile) and s.split == sum(t > L for t in tiles), (len_k, len_q, per_log2, causal, L)
        assert all(t > L for t in tiles[len(tiles) - s.split:])
        assert 1 <= s.parts <= most_parts and (s.parts * L >= s.most or s.parts == most_parts)
        # a whole number of tiles a part, none twice, none left out
        for t in tiles[len(tiles) - s.split:]:
            n = min(s.parts, max(t, 1))
            cut = [t * i // n for i in range(n + 1)]
            assert cut[0] == 0 and cut[-1] == t and min(np.diff(cut)) >= 1


def test_parts_of_mixed_batches_have_room():
    """The length is raised until the parts' sums fit the workspace, whatever the lengths beside one another; it ends; and few tasks of one
    long sequence are split as far as they can be."""
    R, rng = rules(), np.random.default_rng(4)
    for _ in range(300):
        n, units, per_log2, sms, room = int(rng.integers(1, 33)), int(rng.integers(1, 9)), int(rng.integers(4, 9)), 148, int(rng.choice([125, 244]))
        seqs = [(int(np.exp(rng.uniform(0, np.log(300000)))), int(rng.integers(0, 200))) for _ in range(n)]
        if sum(-(-q >> per_log2) if q else 0 for _, q in seqs) * units > sms:
            continue
        total = sum(splitting(k, q, per_log2, True, 1).tiles for k, q in seqs) * units
        L = R.first_length(total, sms)
        assert L >= R.part_limits(1)
        for step in range(200):
            slots = sum(s.split * s.parts for s in (splitting(k, q, per_log2, True, L) for k, q in seqs)) * units
            if slots <= room:
                break
            L += max(1, L // 8)
        assert slots <= room and step < 199
    lone = splitting(100_000, 16, 6, True, R.first_length(782, 148))
    assert (lone.split, lone.parts) == (1, 32)
