"""Host half of the attention calls: refusals before anything is enqueued, tables of rotations, the oracle's own pins, and the rules by
which tasks and ranges are dealt out, restated in Python and held against what they have to cover."""
import ctypes
import math

import numpy as np
import pytest
import torch

from oracle import attention as OA
from paper_2506_04985_b200 import binding as B, rope


@pytest.fixture(scope="module")
def L():
    from paper_2506_04985_b200 import build
    build.build()
    return B.lib()


FAKE, ODD = 0x10000, 0x10008            # never dereferenced: every call fails its checks first
WS = 1 << 26


def cache(**change):
    f = dict(k=FAKE, v=FAKE, k_scale=FAKE, v_scale=FAKE, pages=FAKE, n_pages=4, n_kv=2, page=64, head_dim=128, max_pages=3)
    f.update(change)
    return ctypes.byref(B._KVCacheStruct(**f))


def append(L, **change):
    a = dict(QKV=FAKE, M=5, ld=1024, n_q=4, rope=FAKE, n_pos=100, rot=128, layout=0, cu=FAKE, ctx=FAKE, n=2, cache=cache(), Q=FAKE,
             ld_q=512, K=FAKE, ld_k=256, ws=FAKE, size=WS)
    a.update(change)
    return L.fpt_rope_append(None, *a.values())


def gather(L, **change):
    a = dict(cache=cache(), first=FAKE, cu=FAKE, n=2, M=10, K=FAKE, V=FAKE, ld=256, ws=FAKE, size=WS)
    a.update(change)
    return L.fpt_kv_gather(None, *a.values())


def decode(L, **change):
    a = dict(Q=FAKE, ld_q=512, n_q=4, cache=cache(), lens=FAKE, n=2, scale=0.1, O=FAKE, ld_o=512, lse=FAKE, ws=FAKE, size=WS)
    a.update(change)
    return L.fpt_attn_decode(None, *a.values())


def prompt(L, **change):
    a = dict(Q=FAKE, ld_q=512, Mq=10, K=FAKE, ld_k=256, V=FAKE, ld_v=256, Mk=10, n_q=4, n_kv=2, hd=128, cu_q=FAKE, cu_k=FAKE, n=2,
             causal=1, scale=0.1, O=FAKE, ld_o=512, lse=FAKE, ws=FAKE, size=WS)
    a.update(change)
    return L.fpt_attn_prompt(None, *a.values())


BAD, UNSUPPORTED, ALIGN, ROOM = B.ERR_BAD_ARG, B.ERR_UNSUPPORTED, B.ERR_ALIGNMENT, B.ERR_WORKSPACE


@pytest.mark.parametrize("change,code", [
    (dict(QKV=None), BAD), (dict(rope=None), BAD), (dict(ctx=None), BAD), (dict(Q=None), BAD), (dict(cache=None), BAD),
    (dict(M=0), BAD), (dict(n=0), BAD), (dict(n_q=0), BAD), (dict(n_pos=0), BAD), (dict(layout=2), BAD),
    (dict(ld=1016), BAD), (dict(ld_q=504), BAD), (dict(ld_k=248), BAD), (dict(cu=None, n=6), BAD),
    (dict(rot=0), UNSUPPORTED), (dict(rot=24), UNSUPPORTED), (dict(rot=144), UNSUPPORTED), (dict(n_q=5), UNSUPPORTED),
    (dict(cache=cache(head_dim=96)), UNSUPPORTED), (dict(cache=cache(page=48)), UNSUPPORTED), (dict(cache=cache(page=256)), UNSUPPORTED),
    (dict(cache=cache(n_pages=1 << 30)), UNSUPPORTED), (dict(cache=cache(max_pages=1 << 26)), UNSUPPORTED),
    (dict(n_pos=2 ** 31 - 1), UNSUPPORTED), (dict(cache=cache(v=None)), BAD), (dict(cache=cache(pages=None)), BAD),
    (dict(cache=cache(n_kv=0)), BAD), (dict(cache=cache(n_pages=0)), BAD),
    (dict(ld=1028), ALIGN), (dict(ld_q=516), ALIGN), (dict(ld_k=260), ALIGN), (dict(QKV=ODD), ALIGN), (dict(Q=ODD), ALIGN),
    (dict(K=ODD), ALIGN), (dict(rope=ODD), ALIGN), (dict(cache=cache(k=ODD)), ALIGN), (dict(cache=cache(k_scale=ODD + 1)), ALIGN),
    (dict(cu=FAKE + 2), ALIGN), (dict(ws=None), ROOM), (dict(size=8191), ROOM)])
def test_append_refuses(L, change, code):
    assert append(L, **change) == code


@pytest.mark.parametrize("change,code", [
    (dict(cu=None), BAD), (dict(K=None), BAD), (dict(V=None), BAD), (dict(n=0), BAD), (dict(M=0), BAD), (dict(ld=248), BAD),
    (dict(cache=cache(k=None)), BAD), (dict(cache=None), BAD), (dict(cache=cache(head_dim=32)), UNSUPPORTED),
    (dict(ld=260), ALIGN), (dict(K=ODD), ALIGN), (dict(V=ODD), ALIGN), (dict(first=FAKE + 1), ALIGN), (dict(ws=None), ROOM),
    (dict(size=100), ROOM)])
def test_gather_refuses(L, change, code):
    assert gather(L, **change) == code


@pytest.mark.parametrize("change,code", [
    (dict(Q=None), BAD), (dict(lens=None), BAD), (dict(O=None), BAD), (dict(n=0), BAD), (dict(n_q=0), BAD), (dict(scale=0.0), BAD),
    (dict(scale=-1.0), BAD), (dict(scale=math.nan), BAD), (dict(scale=math.inf), BAD), (dict(ld_q=504), BAD), (dict(ld_o=504), BAD),
    (dict(n_q=5), UNSUPPORTED), (dict(cache=cache(page=8)), UNSUPPORTED), (dict(cache=cache(k_scale=None)), BAD),
    (dict(n=1 << 20, cache=cache(max_pages=1 << 24)), UNSUPPORTED),
    (dict(ld_q=516), ALIGN), (dict(ld_o=516), ALIGN), (dict(Q=ODD), ALIGN), (dict(O=ODD), ALIGN), (dict(lse=FAKE + 2), ALIGN),
    (dict(ws=ODD), ALIGN), (dict(ws=None), ROOM), (dict(size=1 << 20), ROOM)])
def test_decode_refuses(L, change, code):
    assert decode(L, **change) == code


@pytest.mark.parametrize("change,code", [
    (dict(Q=None), BAD), (dict(K=None), BAD), (dict(V=None), BAD), (dict(O=None), BAD), (dict(cu_q=None), BAD), (dict(Mq=0), BAD),
    (dict(Mk=0), BAD), (dict(n=0), BAD), (dict(n_kv=0), BAD), (dict(scale=0.0), BAD), (dict(ld_k=248), BAD), (dict(ld_v=248), BAD),
    (dict(ld_q=504), BAD), (dict(ld_o=504), BAD), (dict(hd=80), UNSUPPORTED), (dict(n_q=3), UNSUPPORTED),
    (dict(Mq=2 ** 31 - 1), UNSUPPORTED), (dict(ld_q=516), ALIGN), (dict(ld_v=260), ALIGN), (dict(V=ODD), ALIGN), (dict(O=ODD), ALIGN),
    (dict(cu_k=FAKE + 2), ALIGN), (dict(ws=None), ROOM), (dict(size=0), ROOM)])
def test_prompt_refuses(L, change, code):
    assert prompt(L, **change) == code


def test_workspace_size_and_words(L):
    size = B.fpt_workspace_bytes(B.OP_ATTN, 1, 1, 1)
    assert size == B.fpt_workspace_bytes(B.OP_ATTN, 5000, 64, 128) and 1 << 20 < size < 1 << 24
    assert "range" in B.strerror(B.ERR_INDEX)


def test_binding_refuses_what_is_not_on_the_device():
    k = torch.zeros((2, 2, 16, 64), dtype=torch.int8)
    s, pages = torch.zeros((2, 2)), torch.zeros((1, 2), dtype=torch.int32)
    c = B.KVCache(k, k.clone(), s, s.clone(), pages)
    q = torch.zeros((1, 128), dtype=torch.bfloat16)
    for call in (lambda: B.fpt_attn_decode(q, c, torch.zeros(1, dtype=torch.int32)),
                 lambda: B.fpt_kv_gather(c, torch.zeros(2, dtype=torch.int32), 1),
                 lambda: B.fpt_attn_prompt(q, q, q, 2, 2, torch.zeros(2, dtype=torch.int32)),
                 lambda: B.fpt_rope_append(torch.zeros((1, 384), dtype=torch.bfloat16), 2, c, torch.zeros((4, 32, 2)),
                                           torch.zeros(1, dtype=torch.int32))):
        with pytest.raises((B.FptError, RuntimeError, AssertionError)):
            call()
    for bad in ((k.float(), k, s, s, pages), (k, k, s, s, pages.long()), (k, k, s[:1], s, pages), (k, k[:, :, ::2], s, s, pages),
                (k.transpose(0, 1), k.transpose(0, 1), s, s, pages)):
        with pytest.raises(ValueError):
            B.KVCache(*bad)


def test_binding_refuses_what_is_no_tensor():
    pages = torch.zeros((1, 2), dtype=torch.int32)
    for bad in ((None,) * 5, (1, "k", None, 2.0, pages)):
        with pytest.raises(ValueError):
            B.KVCache(*bad)
    c, x = B.KVCache.heads(2, 64), torch.zeros((1, 384), dtype=torch.bfloat16)
    ws = torch.zeros(1 << 14, dtype=torch.uint8)
    for call in (lambda: B.fpt_rope_append(None, 2, c, x, x, ws=ws), lambda: B.fpt_attn_decode(3, c, x, ws=ws),
                 lambda: B.fpt_kv_gather(c, [0, 1], 1, ws=ws), lambda: B.fpt_attn_prompt("q", x, x, 2, 2, x, ws=ws),
                 lambda: B.fpt_attn_prompt(x, x, x, 2, 2, x, ws=ws)):
        with pytest.raises(B.FptError) as e:
            call()
        assert e.value.code == B.ERR_BAD_ARG
    with pytest.raises(TypeError):
        B._native().attn_decode(x)


# ------------------------------------------------------------------------------------------------ tables
def test_table_is_right_at_far_positions():
    import fractions
    t = rope.rope_table(3, 128, 500000.0, first=1_000_000)
    f, _ = rope.frequencies(128, 500000.0)
    two_pi = fractions.Fraction("6.283185307179586476925286766559005768394338798750211641949889")
    for row, p in enumerate(range(1_000_000, 1_000_003)):
        for i in (0, 1, 17, 63):
            a = fractions.Fraction(float(f[i])) * p
            a = float(a - two_pi * (a // two_pi))
            assert abs(t[row, i, 0] - math.cos(a)) <= 2.0 ** -24 and abs(t[row, i, 1] - math.sin(a)) <= 2.0 ** -24


def test_scaling_schemes():
    f, one = rope.frequencies(64, 10000.0)
    assert one == 1.0 and f[0] == 1.0 and np.allclose(f[1:] / f[:-1], 10000.0 ** (-2 / 64), rtol=1e-14)
    lin, _ = rope.frequencies(64, 10000.0, "linear", factor=4)
    assert np.array_equal(lin, f / 4)
    ntk, _ = rope.frequencies(64, 10000.0, "ntk", factor=4)
    assert ntk[0] == 1.0 and np.isclose(ntk[-1], f[-1] / 4, rtol=1e-12)
    parts, _ = rope.frequencies(64, 10000.0, "by_parts", factor=8, original=8192, low=1, high=4)
    wave = 2 * math.pi / f
    assert np.array_equal(parts[wave < 8192 / 4], f[wave < 8192 / 4])
    assert np.allclose(parts[wave > 8192], f[wave > 8192] / 8, rtol=1e-14)
    assert ((parts <= f) & (parts >= f / 8 - 1e-18)).all()
    yarn, gain = rope.frequencies(64, 10000.0, "yarn", factor=16, original=4096)
    assert np.isclose(gain, 0.1 * math.log(16) + 1) and yarn[0] == f[0] and np.isclose(yarn[-1], f[-1] / 16)
    t = rope.rope_table(5, 64, scheme="yarn", factor=16, original=4096)
    assert t.shape == (5, 32, 2) and t.dtype == np.float32 and np.allclose((t ** 2).sum(-1), gain ** 2, rtol=1e-6)
    for bad in (dict(rot_dim=63), dict(rot_dim=0), dict(rot_dim=64, factor=0.5, scheme="linear"), dict(rot_dim=64, scheme="other")):
        with pytest.raises(ValueError):
            rope.frequencies(**bad)


# ------------------------------------------------------------------------------------------------ the oracle
def test_oracle_rope_turns_pairs():
    rng = np.random.default_rng(1)
    x = rng.standard_normal((4, 3, 64)).astype(np.float32)
    t = rope.rope_table(4, 32, first=7)
    for inter in (False, True):
        y = OA.rope(x, t, 32, inter)
        a, b = (x[..., 0:32:2], x[..., 1:32:2]) if inter else (x[..., :16], x[..., 16:32])
        z = (a + 1j * b) * (t[:, None, :, 0] + 1j * t[:, None, :, 1])
        c, d = (y[..., 0:32:2], y[..., 1:32:2]) if inter else (y[..., :16], y[..., 16:32])
        assert np.allclose(c, z.real, rtol=2.0 ** -8, atol=1e-6) and np.allclose(d, z.imag, rtol=2.0 ** -8, atol=1e-6)
        assert np.allclose(y[..., 32:], x[..., 32:], rtol=2.0 ** -8)


def test_oracle_append_in_one_go_and_token_by_token():
    """Values come back within half a step of the page's scale; token by token each growth of the scale may add half a step."""
    rng = np.random.default_rng(2)
    v = (rng.standard_normal((50, 2, 64)) * np.linspace(0.2, 3, 50)[:, None, None]).astype(np.float32)
    pages = [3, 0, 5, 1]
    for steps, most in (([50], 0.501), ([1] * 50, 4.0)):
        codes, scale = np.zeros((6, 2, 16, 64), np.int8), np.zeros((6, 2), np.float32)
        at = 0
        for n in steps:
            OA.append(v[at:at + n], codes, scale, pages, at, 16)
            at += n
        back = OA.read(codes, scale, pages, 0, 50, 16)
        step = np.stack([scale[pages[t // 16]] for t in range(50)])[..., None]
        assert (np.abs(back - v) <= most * step).all()
        assert (scale[[2, 4]] == 0).all() and not codes[[2, 4]].any()


def test_oracle_attention_rows_without_keys_and_masks():
    rng = np.random.default_rng(3)
    q, k, v = rng.standard_normal((5, 4, 8)), rng.standard_normal((3, 2, 8)), rng.standard_normal((3, 2, 8))
    o, lse, spread, mass = OA.attend(q, k, v, 0.3, True)
    assert (o[:2] == 0).all() and np.isneginf(lse[:2]).all() and np.isfinite(lse[2:]).all()
    assert np.allclose(o[2], np.repeat(v[0], 2, 0))                          # one key: its value
    v2 = v.copy()
    v2[2] = np.nan                                                           # the last key: only the last query sees it
    o2 = OA.attend(q, k, v2, 0.3, True)[0]
    assert np.allclose(o2[:4], o[:4], rtol=1e-13, atol=1e-15) and np.isnan(o2[4]).all()      # (float64 sums in another order)
    z = 0.3 * np.einsum("qhd,khd->qhk", q, np.repeat(k, 2, 1))
    full = OA.attend(q, k, v, 0.3, False)
    w = np.exp(z) / np.exp(z).sum(-1, keepdims=True)
    assert np.allclose(full[0], np.einsum("qhk,khd->qhd", w, np.repeat(v, 2, 1))) and np.allclose(full[1], np.log(np.exp(z).sum(-1)))


# ------------------------------------------------------------------------------------------------ dealing out
def test_tasks_cover_every_block_that_packed_rows_touch():
    """floor(hi / B) - floor(lo / B) + 2 tasks for rows lo .. hi-1 are enough for the pages they touch at any offset within a page, + 1
    for blocks counted from the first row; a launch of floor(M / B) + (2 or 1) n holds all of them."""
    rng = np.random.default_rng(4)
    for _ in range(300):
        n, block = int(rng.integers(1, 9)), int(rng.choice([16, 32, 64, 128]))
        lens = rng.integers(0, 300, n)
        cu = np.concatenate([[int(rng.integers(0, 50))], lens]).cumsum()
        M = int(cu[-1] + rng.integers(0, 40))
        for extra in (1, 2):
            start = [int(c) // block + extra * s for s, c in enumerate(cu)]
            assert start == sorted(start) and start[-1] <= M // block + extra * n
            for s, length in enumerate(lens):
                offset = int(rng.integers(0, block)) if extra == 2 else 0
                need = 0 if length == 0 else (offset + int(length) - 1) // block + 1
                assert start[s + 1] - start[s] >= need


def test_ranges_of_tiles():
    """The first `longer` ranges have one tile more; a tile's range is found by the same rule the ranges are laid out by."""
    rng = np.random.default_rng(5)
    for _ in range(200):
        total, ctas = int(rng.integers(1, 5000)), int(rng.integers(1, 500))
        ctas = min(ctas, total)
        each, longer = total // ctas, total % ctas
        first = [i * each + min(i, longer) for i in range(ctas + 1)]
        assert first[-1] == total and min(np.diff(first)) >= 1
        edge = longer * (each + 1)
        for x in rng.integers(0, total, 20):
            c = x // (each + 1) if x < edge else longer + (x - edge) // each
            assert first[c] <= x < first[c + 1]


# ------------------------------------------------------------------------------------------------ the source
def test_whole_warps_leave_a_wait_as_one():
    """As in test_waits_cpu.py, for the attention kernels: only the thread that issues the prompt kernel's matrix instructions (roles 2
    and 3 there) waits alone, and nothing waits without a limit."""
    import glob
    import os
    import re
    here = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2506_04985_b200", "csrc")
    seen = 0
    for path in sorted(glob.glob(os.path.join(here, "attn_*.cu"))):
        text = open(path).read()
        name = os.path.basename(path)
        for whole, role in re.findall(r"\bwait_long<(true|false)>\([^;{]*?, (\d+)\)", text):
            seen += 1
            assert (whole == "false") == (name == "attn_prompt.cu" and int(role) in (2, 3)), (name, whole, role)
        assert text.count("wait_long<") == len(re.findall(r"\bwait_long<(?:true|false)>\([^;{]*?, \d+\)", text)), name
        for line in text.splitlines():
            if "mbar_try_wait(" in line:
                assert "globaltimer_ns() - t0 <" in line, (name, line)
        assert "bar.sync" not in text and "__trap" not in text
    assert seen >= 20
