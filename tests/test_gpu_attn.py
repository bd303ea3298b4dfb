"""Rotary positions with the append to the paged 8-bit cache, reading it back, attention over it and of whole prompts,
against the oracle's float64 (and, where a rounding is defined, bit for bit)."""
import math

import numpy as np
import pytest
import torch

from oracle import attention as OA
from paper_2506_04985_b200 import binding as B
from helpers import DEV, bf16_host, guarded_empty, host

pytestmark = pytest.mark.gpu

HALF = 2.0 ** -8           # half a step of bf16, relative


def bf16(rng, *shape, gain=1.0):
    return torch.from_numpy((rng.standard_normal(shape) * gain).astype(np.float32)).to(torch.bfloat16)


def i32(v):
    return torch.tensor(v, dtype=torch.int32, device=DEV)


def offsets(lens):
    return np.concatenate([[0], np.cumsum(lens)]).astype(np.int64)


def table(n_pos, rot, base=500000.0):
    f = base ** (-np.arange(0, rot, 2) / rot)
    a = np.arange(n_pos)[:, None] * f
    return np.stack([np.cos(a), np.sin(a)], -1).astype(np.float32)


def paged(rng, lens, page, n_kv, hd, spare=2, filled=True, width=0):
    """A cache with the pages of the sequences in a random order: (KVCache, page table, codes and scales on the host)."""
    need = [max(1, -(-n // page)) for n in lens]
    n_pages = sum(need) + spare
    order = rng.permutation(n_pages)
    pages = np.full((len(lens), max(max(need), width)), -7, np.int32)      # what no length reaches is not looked at
    at = 0
    for i, n in enumerate(need):
        pages[i, :n] = order[at:at + n]
        at += n
    shape = (n_pages, n_kv, page, hd)
    codes = [rng.integers(-127, 128, shape).astype(np.int8) if filled else np.zeros(shape, np.int8) for _ in "kv"]
    scales = [(rng.uniform(0.5, 4.0, shape[:2]) / 127).astype(np.float32) if filled else np.zeros(shape[:2], np.float32) for _ in "kv"]
    dev = []
    for a in (*codes, *scales):
        t = guarded_empty(a.shape, torch.int8 if a.dtype == np.int8 else torch.float32)
        t.copy_(torch.from_numpy(a))
        dev.append(t)
    return B.KVCache(*dev, i32(pages.tolist())), pages, codes, scales


def workspace():
    return B.new_workspace(B.OP_ATTN, 1, 1, 1)


def close(got, want, bound, what):
    """|got - want| <= bound, infinities and NaN in the same places."""
    got, want = np.asarray(got, np.float64), np.asarray(want, np.float64)
    fine = np.isfinite(want)
    assert (np.isfinite(got) == fine).all(), f"{what}: finite in other places"
    assert np.array_equal(np.isnan(got), np.isnan(want)) and np.array_equal(got[~fine & ~np.isnan(want)], want[~fine & ~np.isnan(want)]), what
    off = np.abs(got[fine] - want[fine]) - np.broadcast_to(bound, want.shape)[fine]
    assert off.size == 0 or off.max() <= 0, f"{what}: {int((off > 0).sum())} of {off.size} off, worst by {off.max():.3g}"


# Bounds of an attention output.  The result's rounding: HALF of it.  A weight's rounding (bf16: HALF, fp16: 2^-11) moves the
# result by at most that share of the weighted mean of |v|.  An exponent is off by the float32 sums' error, at most
# hd * 2^-24 * sum |q k| scale (sums of hd terms in any order; `mass` is the largest such sum), and by a few 2^-24 of itself and of the maximum
# (|z| <= mass); times 1.45 for the change to base 2; the polynomial for powers is 2.7e-6 off, the instruction 2^-22.  A
# weight e^x is off by the same share; numerator and denominator: twice.
def out_bound(o, spread, mass, hd, weight_rounding):
    share = 2 * (1.45 * (hd + 16) * 2.0 ** -24 * mass[..., None] + 3e-6 + 2.0 ** -20)
    return HALF * np.abs(o) + (weight_rounding + share) * (1 + HALF) * spread + 1e-30


def lse_bound(lse, mass, hd):
    return 1.45 * (hd + 16) * 2.0 ** -24 * mass + 4e-6 + 2.0 ** -20 + 2.0 ** -21 * np.abs(np.where(np.isfinite(lse), lse, 0))


# ------------------------------------------------------------------------------------------------ append
APPEND = [
    # hd, page, n_q, n_kv, rot, interleaved, new, ctx
    (128, 64, 32, 8, 128, 0, [1] * 5, [0, 63, 64, 100, 1000]),
    (128, 64, 8, 2, 64, 1, [70, 1, 0, 129, 64], [0, 5, 17, 63, 64]),
    (128, 16, 4, 4, 32, 0, [33, 16, 1, 15], [1, 0, 15, 16]),
    (128, 128, 7, 1, 128, 1, [300, 5], [130, 127]),
    (128, 32, 10, 2, 16, 0, [31, 0, 0, 65], [0, 0, 7, 40]),
    (64, 64, 12, 12, 64, 0, [65, 3, 200], [0, 62, 1]),
    (64, 16, 16, 1, 64, 1, [1, 17, 40], [15, 16, 3]),
    (64, 32, 6, 2, 48, 1, [50, 1], [20, 31]),
    (64, 128, 2, 2, 32, 0, [129, 127, 300], [127, 1, 64]),
]


@pytest.mark.parametrize("hd,page,n_q,n_kv,rot,inter,new,ctx", APPEND)
@pytest.mark.parametrize("odd", [False, True], ids=["plain", "odd values"])
def test_append_matches_the_oracle_bit_for_bit(hd, page, n_q, n_kv, rot, inter, new, ctx, odd):
    rng = np.random.default_rng(hd + page + rot + sum(new) + odd)
    single = all(n == 1 for n in new)
    rows, pad = sum(new), 3
    heads = n_q + 2 * n_kv
    ld = heads * hd + 24
    buf = bf16(rng, rows + pad, ld)
    if odd:
        x = buf[:rows, :heads * hd].view(rows, heads, hd)
        x[rows // 2, n_q:, 5] = math.inf
        x[0, n_q:, hd - 1] = -math.inf
        x[rows - 1, n_q:, rot // 2] = math.nan
        x[:, n_q + n_kv] = 0                             # a value head of zeros
        x[0, n_q + n_kv, 3] = 1e-38                       # ... but for one whose page's scale is below 2^-126
    cache, pages, codes, scales = paged(rng, [c + n for c, n in zip(ctx, new)], page, n_kv, hd)
    if odd:
        for s in scales:
            s[:, 0] = 0                                  # pages that hold zeros so far
        cache.k_scale.copy_(torch.from_numpy(scales[0])), cache.v_scale.copy_(torch.from_numpy(scales[1]))
    tab = table(max(c + n for c, n in zip(ctx, new)), rot)
    qkv = buf.to(DEV)[:, :heads * hd]
    Q = guarded_empty((rows + pad, n_q * hd), torch.bfloat16)
    K = guarded_empty((rows + pad, n_kv * hd), torch.bfloat16)
    Q.fill_(7.0), K.fill_(7.0)
    ws = workspace()
    cu = offsets(new)
    B.fpt_rope_append(qkv, n_q, cache, torch.from_numpy(tab).to(DEV), i32(ctx), cu_new=None if single else i32(cu.tolist()),
                      layout=B.ROPE_INTERLEAVED if inter else B.ROPE_HALF, Q=Q, K=K, ws=ws)
    assert B.fpt_check_status(ws) == B.OK
    x = buf[:, :heads * hd].float().numpy().reshape(rows + pad, heads, hd)
    for i, (n, c) in enumerate(zip(new, ctx)):
        a = cu[i]
        with np.errstate(invalid="ignore"):
            qk = OA.rope(x[a:a + n, :n_q + n_kv], tab[c:c + n], rot, inter)
        assert np.array_equal(bf16_host(Q)[a:a + n], qk[:, :n_q].reshape(n, n_q * hd), equal_nan=True)
        assert np.array_equal(bf16_host(K)[a:a + n], qk[:, n_q:].reshape(n, n_kv * hd), equal_nan=True)
        if n:
            OA.append(qk[:, n_q:], codes[0], scales[0], pages[i], c, page)
            OA.append(x[a:a + n, n_q + n_kv:], codes[1], scales[1], pages[i], c, page)
    for got, want in zip((cache.k_scale, cache.v_scale, cache.k, cache.v), (*scales, *codes)):
        assert np.array_equal(host(got), want)            # pages that nothing was added to among them
    assert (bf16_host(Q)[rows:] == 7).all() and (bf16_host(K)[rows:] == 7).all()


def test_append_token_by_token_grows_the_scale_as_the_oracle_does():
    rng = np.random.default_rng(5)
    n_q, n_kv, hd, page, n = 8, 2, 128, 16, 37
    cache, pages, codes, scales = paged(rng, [n], page, n_kv, hd)
    tab = table(n, hd)
    qkv = bf16(rng, n, (n_q + 2 * n_kv) * hd) * torch.linspace(0.1, 5, n)[:, None].to(torch.bfloat16)
    ws, tabd, dev = workspace(), torch.from_numpy(tab).to(DEV), qkv.to(DEV)
    x = qkv.float().numpy().reshape(n, -1, hd)
    for t in range(n):
        B.fpt_rope_append(dev[t:t + 1], n_q, cache, tabd, i32([t]), ws=ws)
        k = OA.rope(x[t:t + 1, n_q:n_q + n_kv], tab[t:t + 1], hd, False)
        OA.append(k, codes[0], scales[0], pages[0], t, page)
        OA.append(x[t:t + 1, n_q + n_kv:], codes[1], scales[1], pages[0], t, page)
    assert B.fpt_check_status(ws) == B.OK
    for got, want in zip((cache.k_scale, cache.v_scale, cache.k, cache.v), (*scales, *codes)):
        assert np.array_equal(host(got), want)


def test_rotation_alone_and_in_place():
    rng = np.random.default_rng(6)
    n_q, n_kv, hd, new, ctx = 6, 2, 64, [3, 130], [10, 0]
    x = bf16(rng, sum(new), (n_q + 2 * n_kv) * hd)
    tab = table(140, 32)
    dev, ws = x.to(DEV), workspace()
    B.fpt_rope_append(dev, n_q, B.KVCache.heads(n_kv, hd), torch.from_numpy(tab).to(DEV), i32(ctx), cu_new=i32([0, 3, 133]),
                      Q=dev[:, :n_q * hd], K=dev[:, n_q * hd:(n_q + n_kv) * hd], ws=ws)
    assert B.fpt_check_status(ws) == B.OK
    got, want = bf16_host(dev).reshape(133, -1, hd), x.float().numpy().reshape(133, -1, hd)
    pos = np.concatenate([np.arange(10, 13), np.arange(130)])
    want[:, :n_q + n_kv] = OA.rope(want[:, :n_q + n_kv], tab[pos], 32, False)
    assert np.array_equal(got, want)


# ------------------------------------------------------------------------------------------------ gather
@pytest.mark.parametrize("hd,page,n_kv,first,count", [
    (128, 64, 8, [0, 3, 64], [64, 200, 1]), (128, 16, 1, [15, 0], [2, 0]), (64, 32, 3, [0, 31, 5], [1, 33, 100]),
    (64, 128, 12, [100], [300]), (128, 128, 2, [0, 0, 127], [129, 0, 1])])
def test_gather_gives_the_held_values(hd, page, n_kv, first, count):
    rng = np.random.default_rng(7)
    cache, pages, codes, scales = paged(rng, [f + c for f, c in zip(first, count)], page, n_kv, hd)
    rows, ws = sum(count) + 2, workspace()
    wide = guarded_empty((rows, 2 * n_kv * hd), torch.bfloat16)
    wide.fill_(7.0)
    K, V = wide[:, :n_kv * hd], wide[:, n_kv * hd:]
    B.fpt_kv_gather(cache, i32(offsets(count).tolist()), rows, first=i32(first), K=K, V=V, ws=ws)
    assert B.fpt_check_status(ws) == B.OK
    for got, c, s in ((K, codes[0], scales[0]), (V, codes[1], scales[1])):
        want = np.concatenate([OA.read(c, s, pages[i], f, n, page) for i, (f, n) in enumerate(zip(first, count))])
        want = torch.from_numpy(want).to(torch.bfloat16).float().numpy().reshape(rows - 2, -1)
        assert np.array_equal(bf16_host(got)[:-2], want) and (bf16_host(got)[-2:] == 7).all()


# ------------------------------------------------------------------------------------------------ one token
DECODE = [
    # hd, page, n_q, n_kv, lengths
    (128, 64, 32, 8, [1]),
    (128, 64, 32, 8, [1000]),
    (128, 64, 32, 8, [0, 1, 63, 64, 65, 127, 128, 129, 700]),
    (128, 16, 4, 4, [17, 0, 5, 333, 16]),
    (128, 32, 7, 1, [2000, 33, 1]),
    (128, 128, 10, 2, [129, 1, 0, 257]),
    (128, 64, 16, 1, [555, 64]),                 # 16 heads on one
    (128, 64, 40, 2, [300, 20]),                 # 20: two blocks, the second of four
    (128, 16, 64, 1, [77]),                      # 64: four blocks
    (64, 64, 12, 12, [0, 2500, 1, 64]),
    (64, 16, 9, 3, [100, 47, 15]),
    (64, 32, 24, 2, [65, 400]),
    (64, 128, 8, 1, [1000, 128]),
]


def decode_case(rng, hd, page, n_q, n_kv, lens, gain=1.0):
    cache, pages, codes, scales = paged(rng, lens, page, n_kv, hd)
    q = bf16(rng, len(lens), n_q * hd, gain=gain)
    return cache, pages, codes, scales, q


def check_decode(got, lse, lens, pages, codes, scales, q, n_q, hd, page, scale):
    for i, n in enumerate(lens):
        k, v = (OA.read(codes[j], scales[j], pages[i], 0, n, page) for j in (0, 1))
        o, z, spread, mass = OA.attend(q[i].float().numpy().reshape(1, n_q, hd), k, v, scale, False)
        close(bf16_host(got)[i].reshape(1, n_q, hd), o, out_bound(o, spread, mass, hd, 2.0 ** -11), f"sequence {i} of {n}")
        if lse is not None:
            close(host(lse)[i][None], z, lse_bound(z, mass, hd), f"lse of sequence {i}")


@pytest.mark.parametrize("hd,page,n_q,n_kv,lens", DECODE)
def test_decode(hd, page, n_q, n_kv, lens):
    rng = np.random.default_rng(sum(lens) + hd)
    cache, pages, codes, scales, q = decode_case(rng, hd, page, n_q, n_kv, lens)
    ws = workspace()
    o, lse = B.fpt_attn_decode(q.to(DEV), cache, i32(lens), want_lse=True, ws=ws)
    assert B.fpt_check_status(ws) == B.OK
    check_decode(o, lse, lens, pages, codes, scales, q, n_q, hd, page, hd ** -0.5)
    again, _ = B.fpt_attn_decode(q.to(DEV), cache, i32(lens), ws=ws)       # the counters are back where they were
    assert torch.equal(o.view(torch.int16), again.view(torch.int16))


def test_decode_sharp_weights_and_uneven_scales():
    """One key far above the others, maxima that keep growing along the sequence, pages whose scales lie far apart, a page of zeros."""
    rng = np.random.default_rng(9)
    hd, page, n_q, n_kv, lens = 128, 32, 8, 2, [900, 64]
    cache, pages, codes, scales, q = decode_case(rng, hd, page, n_q, n_kv, lens, gain=3.0)
    for p, i in enumerate(pages[0]):
        scales[0][i] *= 1.0 + 0.2 * p
        scales[1][i] *= 10.0 ** (p % 7 - 3)
    scales[1][pages[0][3]] = 0
    codes[1][pages[0][3]] = 0
    cache.k_scale.copy_(torch.from_numpy(scales[0])), cache.v_scale.copy_(torch.from_numpy(scales[1]))
    cache.v.copy_(torch.from_numpy(codes[1]))
    o, lse = B.fpt_attn_decode(q.to(DEV), cache, i32(lens), want_lse=True)
    check_decode(o, lse, lens, pages, codes, scales, q, n_q, hd, page, hd ** -0.5)


def test_decode_queries_of_any_size():
    rng = np.random.default_rng(10)
    hd, page, n_q, n_kv, lens = 64, 64, 4, 2, [200] * 4
    cache, pages, codes, scales, q = decode_case(rng, hd, page, n_q, n_kv, lens)
    q[1] *= 1e-30
    q[2] = 0
    q[3] *= 1e6
    o, lse = B.fpt_attn_decode(q.to(DEV), cache, i32(lens), scale=1e-5, want_lse=True)
    check_decode(o, lse, lens, pages, codes, scales, q, n_q, hd, page, 1e-5)


def test_decode_rows_in_wider_buffers():
    rng = np.random.default_rng(11)
    hd, page, n_q, n_kv, lens = 128, 64, 8, 2, [70, 300, 5]
    cache, pages, codes, scales, q = decode_case(rng, hd, page, n_q, n_kv, lens)
    wide = torch.full((3, n_q * hd + 40), 5.0, dtype=torch.bfloat16)
    wide[:, :n_q * hd] = q
    out = guarded_empty((3, n_q * hd + 8), torch.bfloat16)
    out.fill_(7.0)
    o, _ = B.fpt_attn_decode(wide.to(DEV)[:, :n_q * hd], cache, i32(lens), O=out[:, :n_q * hd])
    check_decode(o, None, lens, pages, codes, scales, q, n_q, hd, page, hd ** -0.5)
    assert (bf16_host(out)[:, n_q * hd:] == 7).all()


def test_decode_many_sequences():
    """More sequences than one look at the lengths takes, more rows than CTAs."""
    rng = np.random.default_rng(12)
    hd, page, n_q, n_kv = 64, 16, 4, 4
    lens = [int(n) for n in rng.integers(0, 150, 333)]
    cache, pages, codes, scales, q = decode_case(rng, hd, page, n_q, n_kv, lens)
    o, lse = B.fpt_attn_decode(q.to(DEV), cache, i32(lens), want_lse=True)
    check_decode(o, lse, lens, pages, codes, scales, q, n_q, hd, page, hd ** -0.5)


def test_decode_page_out_of_range_is_recorded_and_spares_the_others():
    rng = np.random.default_rng(13)
    hd, page, n_q, n_kv, lens = 128, 16, 4, 2, [100, 40, 64]
    cache, pages, codes, scales, q = decode_case(rng, hd, page, n_q, n_kv, lens)
    cache.pages[1, 1] = 1 << 30
    ws = workspace()
    o, _ = B.fpt_attn_decode(q.to(DEV), cache, i32(lens), ws=ws)
    assert B.fpt_check_status(ws) == B.ERR_INDEX
    check_decode(o[0:1], None, lens[:1], pages[:1], codes, scales, q[:1], n_q, hd, page, hd ** -0.5)
    check_decode(o[2:3], None, lens[2:], pages[2:], codes, scales, q[2:], n_q, hd, page, hd ** -0.5)
    B.lib().fpt_reset_status(B._stream(), B._ptr(ws))
    cache.pages[1, 1] = int(pages[1, 1])
    B.fpt_attn_decode(q.to(DEV), cache, i32([100, 40, 1 << 28]), ws=ws)       # longer than its pages: cut to them
    assert B.fpt_check_status(ws) == B.ERR_INDEX


# ------------------------------------------------------------------------------------------------ prompts
PROMPT = [
    # hd, n_q, n_kv, len_q, len_k (None: the same), causal
    (128, 32, 8, [1], None, True),
    (128, 4, 1, [130], None, True),
    (128, 4, 1, [64, 1, 127, 65, 128, 3], None, True),
    (128, 8, 8, [129, 300], None, True),
    (128, 7, 1, [200, 13], None, True),
    (128, 12, 2, [100, 0, 50], None, True),
    (128, 16, 1, [40, 9], None, True),
    (128, 2, 2, [40, 300, 5], [300, 300, 700], True),        # chunks behind prefixes
    (128, 4, 2, [100, 260, 7, 3], [20, 0, 3, 130], True),    # more queries than keys, no keys
    (128, 4, 2, [100, 3], [333, 128], False),
    (64, 24, 4, [257, 31], None, True),
    (64, 3, 3, [128, 256, 511], None, True),
    (64, 8, 1, [77, 5], [600, 129], True),
    (64, 8, 2, [0, 300], [10, 200], False),
    (128, 4, 4, [1100], None, True),                          # the ring of tiles more than once around
    (64, 4, 4, [1300], [1700], True),
]


def prompt_case(rng, hd, n_q, n_kv, len_q, len_k, pad=5):
    return (bf16(rng, sum(len_q) + pad, n_q * hd), bf16(rng, sum(len_k) + pad, n_kv * hd, gain=1.5),
            bf16(rng, sum(len_k) + pad, n_kv * hd))


def check_prompt(got, lse, q, k, v, n_q, n_kv, hd, len_q, len_k, causal, scale=None):
    a, b = offsets(len_q), offsets(len_k)
    for i in range(len(len_q)):
        args = [t.float().numpy()[x[i]:x[i + 1]].reshape(x[i + 1] - x[i], t.shape[1] // hd, hd) for t, x in ((q, a), (k, b), (v, b))]
        o, z, spread, mass = OA.attend(*args, hd ** -0.5 if scale is None else scale, causal)
        close(bf16_host(got)[a[i]:a[i + 1]].reshape(o.shape), o, out_bound(o, spread, mass, hd, HALF), f"sequence {i}")
        if lse is not None:
            close(host(lse)[a[i]:a[i + 1]], z, lse_bound(z, mass, hd), f"lse of sequence {i}")


@pytest.mark.parametrize("hd,n_q,n_kv,len_q,len_k,causal", PROMPT)
def test_prompt(hd, n_q, n_kv, len_q, len_k, causal):
    same, len_k = len_k is None, len_k or len_q
    rng = np.random.default_rng(sum(len_q) + hd + n_q)
    q, k, v = prompt_case(rng, hd, n_q, n_kv, len_q, len_k)
    k[sum(len_k):] = math.nan                            # rows behind the last sequence
    v[sum(len_k):] = math.inf
    rows = sum(len_q)
    out = guarded_empty(q.shape, torch.bfloat16)
    out.fill_(7.0)
    ws = workspace()
    _, lse = B.fpt_attn_prompt(q.to(DEV), k.to(DEV), v.to(DEV), n_q, n_kv, i32(offsets(len_q).tolist()),
                               cu_k=None if same else i32(offsets(len_k).tolist()), causal=causal, want_lse=True, O=out, ws=ws)
    assert B.fpt_check_status(ws) == B.OK
    check_prompt(out, lse, q, k, v, n_q, n_kv, hd, len_q, len_k, causal)
    assert (bf16_host(out)[rows:] == 7).all()


def test_prompt_from_one_buffer():
    """Queries, keys and values as places of one projection's rows; the output in a wider buffer."""
    rng = np.random.default_rng(21)
    hd, n_q, n_kv, lens = 128, 8, 2, [150, 33]
    x = bf16(rng, sum(lens), (n_q + 2 * n_kv) * hd + 16)
    d = x.to(DEV)
    cut = [(0, n_q * hd), (n_q * hd, (n_q + n_kv) * hd), ((n_q + n_kv) * hd, (n_q + 2 * n_kv) * hd)]
    out = guarded_empty((sum(lens), n_q * hd + 8), torch.bfloat16)
    out.fill_(7.0)
    B.fpt_attn_prompt(*(d[:, a:b] for a, b in cut), n_q, n_kv, i32([0, 150, 183]), O=out[:, :n_q * hd])
    check_prompt(out[:, :n_q * hd], None, *(x[:, a:b] for a, b in cut), n_q, n_kv, hd, lens, lens, True)
    assert (bf16_host(out)[:, n_q * hd:] == 7).all()


@pytest.mark.parametrize("hd", [64, 128])
def test_prompt_maxima_that_grow_and_sharp_weights(hd):
    """Scores that climb along the keys: every tile renews the maximum and turns the sums in tensor memory down."""
    rng = np.random.default_rng(22)
    n_q, n_kv, lens = 2, 1, [700]
    q, k, v = prompt_case(rng, hd, n_q, n_kv, lens, lens, pad=0)
    q.fill_(1.0)
    k.copy_((torch.linspace(-1, 1, 700)[:, None] * 40 / hd ** 0.5 + 0.02 * torch.randn(700, hd, generator=torch.Generator().manual_seed(1))).to(torch.bfloat16))
    o, lse = B.fpt_attn_prompt(q.to(DEV), k.to(DEV), v.to(DEV), n_q, n_kv, i32([0, 700]), want_lse=True)
    check_prompt(o, lse, q, k, v, n_q, n_kv, hd, lens, lens, True)


@pytest.mark.parametrize("hd", [64, 128])
def test_prompt_odd_values_reach_only_who_sees_them(hd):
    """Infinities and NaN among keys and values: queries in front of them, and other sequences, are untouched."""
    rng = np.random.default_rng(23)
    n_q, n_kv, lens = 4, 2, [200, 70, 30]
    q, k, v = prompt_case(rng, hd, n_q, n_kv, lens, lens, pad=0)
    v[150, 3] = math.inf
    v[190, 3] = -math.inf
    v[199, hd + 1] = math.nan
    k[180, hd:] = math.nan                               # the second key head
    v[260, :] = math.nan
    k[205, 0] = math.inf
    o, lse = B.fpt_attn_prompt(q.to(DEV), k.to(DEV), v.to(DEV), n_q, n_kv, i32(offsets(lens).tolist()), want_lse=True)
    got = bf16_host(o)
    # the oracle leaves hidden keys and values out row by row; where a value that is not finite is seen, so is the result
    a = offsets(lens)
    for i in range(3):
        args = [t.float().numpy()[a[i]:a[i + 1]].reshape(lens[i], -1, hd) for t in (q, k, v)]
        want, _, spread, mass = OA.attend(*args, hd ** -0.5, True)
        mine = got[a[i]:a[i + 1]].reshape(want.shape)
        fine = np.isfinite(want)
        assert (np.isfinite(mine) == fine).all(), i
        assert (np.abs(mine - want)[fine] <= out_bound(want, spread, mass, hd, HALF)[fine]).all(), i


def test_prompt_offsets_out_of_range_are_recorded():
    rng = np.random.default_rng(24)
    q, k, v = (t.to(DEV) for t in prompt_case(rng, 64, 2, 1, [100], [100], pad=0))
    for cu in ([0, 101], [0, -5], [-3, 40], [50, 20]):
        ws = workspace()
        out = guarded_empty(q.shape, torch.bfloat16)
        B.fpt_attn_prompt(q, k, v, 2, 1, i32(cu), O=out, ws=ws)
        B.fpt_attn_prompt(q, k, v, 2, 1, i32([0, 100]), cu_k=i32(cu), O=out, ws=ws)
        assert B.fpt_check_status(ws) == B.ERR_INDEX, cu


# ------------------------------------------------------------------------------------------------ together
@pytest.mark.parametrize("hd,page,inter", [(128, 64, False), (64, 16, True)])
def test_a_prompt_in_chunks_and_single_tokens_agree(hd, page, inter):
    """The run of a server: a prompt in two chunks (append, prefix in 16 bits, attention), then tokens one at a time."""
    rng = np.random.default_rng(31)
    n_q, n_kv, lens, steps = 8, 2, [90, 33], 3
    total = [n + steps for n in lens]
    cache, pages, codes, scales = paged(rng, total, page, n_kv, hd, filled=False)
    tab = table(max(total), hd)
    tabd, ws = torch.from_numpy(tab).to(DEV), workspace()
    layout = B.ROPE_INTERLEAVED if inter else B.ROPE_HALF
    x = [bf16(rng, n, (n_q + 2 * n_kv) * hd) for n in total]
    have = [0, 0]
    plan = [[50, 20], [40, 13]] + [[1, 1]] * steps
    for new in plan:
        rows = torch.cat([x[i][have[i]:have[i] + n] for i, n in enumerate(new)]).to(DEV)
        ends = [h + n for h, n in zip(have, new)]
        cu = i32(offsets(new).tolist())
        single = new == [1, 1]
        q, _ = B.fpt_rope_append(rows, n_q, cache, tabd, i32(have), cu_new=None if single else cu, layout=layout, ws=ws)
        if single:
            o, _ = B.fpt_attn_decode(q, cache, i32(ends), ws=ws)
        else:
            cu_k = i32(offsets(ends).tolist())
            k, v = B.fpt_kv_gather(cache, cu_k, sum(ends), ws=ws)
            o, _ = B.fpt_attn_prompt(q, k, v, n_q, n_kv, cu, cu_k=cu_k, ws=ws)
        assert B.fpt_check_status(ws) == B.OK
        a = offsets(new)
        for i, n in enumerate(new):
            y = x[i].float().numpy().reshape(total[i], -1, hd)
            qk = OA.rope(y[have[i]:ends[i], :n_q + n_kv], tab[have[i]:ends[i]], hd, inter)
            OA.append(qk[:, n_q:], codes[0], scales[0], pages[i], have[i], page)
            OA.append(y[have[i]:ends[i], n_q + n_kv:], codes[1], scales[1], pages[i], have[i], page)
            kk, vv = (OA.read(codes[j], scales[j], pages[i], 0, ends[i], page) for j in (0, 1))
            if not single:
                kk, vv = (torch.from_numpy(t).to(torch.bfloat16).float().numpy() for t in (kk, vv))
            want, _, spread, mass = OA.attend(qk[:, :n_q], kk, vv, hd ** -0.5, True)
            close(bf16_host(o)[a[i]:a[i + 1]].reshape(want.shape), want,
                  out_bound(want, spread, mass, hd, 2.0 ** -11 if single else HALF), f"sequence {i} at {have[i]}")
        have = ends
    for got, want in zip((cache.k_scale, cache.v_scale, cache.k, cache.v), (*scales, *codes)):
        assert np.array_equal(host(got), want)


# ------------------------------------------------------------------------------------------------ as a program holds them
def test_the_attention_block_from_projection_to_projection():
    """fpt_decoder_attn_qkv, then the attention of a prompt, then a decode step of the same sequences, fpt_decoder_attn_out behind each: the
    calls chained on one stream and one workspace give what each gives with a wait in between."""
    from paper_2506_04985_b200 import synth
    d, n_q, n_kv, hd, page, lens = 512, 8, 2, 64, 32, [37, 5]
    n_qkv = (n_q + 2 * n_kv) * hd
    wq, sq, _ = B.fpt_quantize_weights(synth.weights(n_qkv, d, 0.05, 1, "block/qkv").to(DEV))
    wo, so, _ = B.fpt_quantize_weights(synth.weights(d, n_q * hd, 0.05, 1, "block/o").to(DEV))
    qp_in, qp_ap = B.QParams(4, True, 0.4, 0), B.QParams(4, True, 0.1, 0)
    total = sum(lens)
    x = synth.activations(total, d, 1, "block/x", law="normal").to(DEV)
    x1 = synth.activations(2, d, 2, "block/x1", law="normal").to(DEV)
    tab = torch.from_numpy(table(64, hd)).to(DEV)
    room = max(B.fpt_workspace_bytes(B.OP_ATTN, 1, 1, 1), B.fpt_workspace_bytes(B.OP_LINEAR, total, n_qkv, d),
               B.fpt_workspace_bytes(B.OP_LINEAR, 2, n_qkv, d))

    def run(wait):
        stop = torch.cuda.synchronize if wait else (lambda: None)
        ws = guarded_empty((room,), torch.uint8)
        B.lib().fpt_reset_status(B._stream(), B._ptr(ws))
        rng = np.random.default_rng(77)
        cache, *_ = paged(rng, [n + 1 for n in lens], page, n_kv, hd, filled=False)
        cu, ctx0, ctx1, ends = i32([0, 37, 42]), i32([0, 0]), i32(lens), i32([n + 1 for n in lens])
        outs = []
        qkv, s_n, r = B.fpt_decoder_attn_qkv(x, wq, sq, qp_in, ws=ws); stop()
        q, k = B.fpt_rope_append(qkv, n_q, cache, tab, ctx0, cu_new=cu, want_k=True, ws=ws); stop()
        o, _ = B.fpt_attn_prompt(q, k, qkv[:, (n_q + n_kv) * hd:], n_q, n_kv, cu, ws=ws); stop()
        outs += [o, B.fpt_decoder_attn_out(o, wo, so, qp_ap, s_n, X=x, r=r, ws=ws)]; stop()
        qkv, s_n, r = B.fpt_decoder_attn_qkv(x1, wq, sq, qp_in, ws=ws); stop()
        q, _ = B.fpt_rope_append(qkv, n_q, cache, tab, ctx1, ws=ws); stop()
        o, _ = B.fpt_attn_decode(q, cache, ends, ws=ws); stop()
        outs += [o, B.fpt_decoder_attn_out(o, wo, so, qp_ap, s_n, X=x1, r=r, ws=ws)]
        assert B.fpt_check_status(ws) == B.OK
        return [t.clone() for t in outs]

    a, b = run(True), run(False)
    for u, v in zip(a, b):
        assert torch.equal(u.view(torch.int16), v.view(torch.int16)) and torch.isfinite(u.float()).all()


def test_decode_step_in_a_graph_follows_the_lengths_on_the_device():
    """One captured step replayed while contexts grow: positions, lengths and pages are read from the device each time; so with
    launches that wait for one another in the stream, and without."""
    rng = np.random.default_rng(41)
    hd, page, n_q, n_kv, steps, start = 128, 16, 8, 2, 20, [0, 14, 63]
    total = [s + steps for s in start]
    x = bf16(rng, steps, 3, (n_q + 2 * n_kv) * hd)
    tab = table(max(total), hd)
    tabd, ws = torch.from_numpy(tab).to(DEV), workspace()
    for early in (True, False):
        rng = np.random.default_rng(42)
        cache, pages, codes, scales = paged(rng, total, page, n_kv, hd)
        was = B.fpt_set_programmatic_launch(early)
        try:
            row, ctx, ends = x[0].to(DEV), i32(start), i32([s + 1 for s in start])
            Q, O = (guarded_empty((3, n_q * hd), torch.bfloat16) for _ in range(2))

            def step():
                B.fpt_rope_append(row, n_q, cache, tabd, ctx, Q=Q, ws=ws)
                B.fpt_attn_decode(Q, cache, ends, O=O, ws=ws)

            keep = [t.clone() for t in (cache.k, cache.v, cache.k_scale, cache.v_scale)]
            stream = torch.cuda.Stream()
            with torch.cuda.stream(stream):
                step()                                       # (kernels are loaded outside the capture)
                torch.cuda.synchronize()
                for t, old in zip((cache.k, cache.v, cache.k_scale, cache.v_scale), keep):
                    t.copy_(old)
                g = torch.cuda.CUDAGraph()
                with torch.cuda.graph(g, stream=stream):
                    step()
                for t in range(steps):
                    row.copy_(x[t]), ctx.copy_(i32([s + t for s in start])), ends.copy_(i32([s + t + 1 for s in start]))
                    g.replay()
                    stream.synchronize()
                    for i in range(3):
                        y = x[t, i].float().numpy().reshape(1, -1, hd)
                        qk = OA.rope(y[:, :n_q + n_kv], tab[start[i] + t:start[i] + t + 1], hd, False)
                        OA.append(qk[:, n_q:], codes[0], scales[0], pages[i], start[i] + t, page)
                        OA.append(y[:, n_q + n_kv:], codes[1], scales[1], pages[i], start[i] + t, page)
                    if t % 7 == 0 or t == steps - 1:
                        q = Q.float().cpu().to(torch.bfloat16)
                        check_decode(O, None, [s + t + 1 for s in start], pages, codes, scales, q, n_q, hd, page, hd ** -0.5)
                assert B.fpt_check_status(ws) == B.OK
            for got, want in zip((cache.k_scale, cache.v_scale, cache.k, cache.v), (*scales, *codes)):
                assert np.array_equal(host(got), want)
        finally:
            B.fpt_set_programmatic_launch(was)


def test_two_streams_with_a_workspace_each():
    rng = np.random.default_rng(43)
    hd, page, n_q, n_kv, lens = 128, 64, 8, 2, [3000, 1500]
    cache, pages, codes, scales, q = decode_case(rng, hd, page, n_q, n_kv, lens)
    qd, ld = q.to(DEV), i32(lens)
    want, _ = B.fpt_attn_decode(qd, cache, ld)
    torch.cuda.synchronize()
    streams, wss, outs = [torch.cuda.Stream() for _ in range(2)], [workspace() for _ in range(2)], []
    torch.cuda.synchronize()
    for k in range(40):
        with torch.cuda.stream(streams[k % 2]):
            outs.append(B.fpt_attn_decode(qd, cache, ld, ws=wss[k % 2])[0])
    torch.cuda.synchronize()
    for o in outs:
        assert torch.equal(o.view(torch.int16), want.view(torch.int16))


def test_prompt_gives_the_same_bits_each_time():
    """Tasks go to whichever CTA is free; what a task computes does not depend on it."""
    rng = np.random.default_rng(44)
    hd, n_q, n_kv, lens = 128, 8, 2, [int(n) for n in rng.integers(1, 400, 40)]
    q, k, v = (t.to(DEV) for t in prompt_case(rng, hd, n_q, n_kv, lens, lens, pad=0))
    cu = i32(offsets(lens).tolist())
    first, _ = B.fpt_attn_prompt(q, k, v, n_q, n_kv, cu)
    for _ in range(5):
        o, _ = B.fpt_attn_prompt(q, k, v, n_q, n_kv, cu)
        assert torch.equal(o.view(torch.int16), first.view(torch.int16))


@pytest.mark.parametrize("n", [32, 33, 128, 129, 300])
def test_prompt_many_sequences(n):
    """As many as a warp's lanes, as are held in registers, and more: each way of finding a task; empty ones among them."""
    rng = np.random.default_rng(n)
    hd, n_q, n_kv = 64, 4, 2
    lens = [int(x) for x in rng.integers(0, 90, n)]
    pre = [int(x) for x in rng.integers(0, 60, n)]
    len_k = [a + b if i % 3 else a for i, (a, b) in enumerate(zip(lens, pre))]
    q, k, v = prompt_case(rng, hd, n_q, n_kv, lens, len_k)
    ws = workspace()
    o, lse = B.fpt_attn_prompt(q.to(DEV), k.to(DEV), v.to(DEV), n_q, n_kv, i32(offsets(lens).tolist()), cu_k=i32(offsets(len_k).tolist()),
                               want_lse=True, ws=ws)
    assert B.fpt_check_status(ws) == B.OK
    check_prompt(o, lse, q, k, v, n_q, n_kv, hd, lens, len_k, True)


def test_append_and_gather_many_sequences():
    rng = np.random.default_rng(45)
    hd, page, n_q, n_kv, n = 64, 16, 2, 1, 400
    new, ctx = [int(x) for x in rng.integers(0, 40, n)], [int(x) for x in rng.integers(0, 40, n)]
    cache, pages, codes, scales = paged(rng, [a + b for a, b in zip(new, ctx)], page, n_kv, hd)
    x, tab, ws = bf16(rng, sum(new), (n_q + 2 * n_kv) * hd), table(80, hd), workspace()
    cu = offsets(new)
    B.fpt_rope_append(x.to(DEV), n_q, cache, torch.from_numpy(tab).to(DEV), i32(ctx), cu_new=i32(cu.tolist()), ws=ws)
    ends = [a + b for a, b in zip(new, ctx)]
    K, V = B.fpt_kv_gather(cache, i32(offsets(ends).tolist()), sum(ends), ws=ws)
    assert B.fpt_check_status(ws) == B.OK
    y = x.float().numpy().reshape(-1, n_q + 2 * n_kv, hd)
    for i in range(n):
        if new[i]:
            part = y[cu[i]:cu[i + 1]]
            k = OA.rope(part[:, n_q:n_q + n_kv], tab[ctx[i]:ends[i]], hd, False)
            OA.append(k, codes[0], scales[0], pages[i], ctx[i], page)
            OA.append(part[:, n_q + n_kv:], codes[1], scales[1], pages[i], ctx[i], page)
    for got, want in zip((cache.k_scale, cache.v_scale, cache.k, cache.v), (*scales, *codes)):
        assert np.array_equal(host(got), want)
    for got, j in ((K, 0), (V, 1)):
        want = np.concatenate([OA.read(codes[j], scales[j], pages[i], 0, e, page) for i, e in enumerate(ends)])
        assert np.array_equal(bf16_host(got), torch.from_numpy(want).to(torch.bfloat16).float().numpy().reshape(got.shape))


def test_cache_offsets_beyond_32_bits():
    """A sequence in the last pages of a cache whose codes take more than 4 GiB."""
    hd, page, n_q, n_kv, n_pages, n = 128, 64, 8, 8, 70_000, 200
    if torch.cuda.mem_get_info()[0] < 16 << 30:
        pytest.skip("needs 10 GB")
    k, v = (torch.zeros((n_pages, n_kv, page, hd), dtype=torch.int8, device=DEV) for _ in range(2))
    ks, vs = (torch.zeros((n_pages, n_kv), device=DEV) for _ in range(2))
    pages = np.array([[n_pages - 1, n_pages - 3, 1, n_pages - 2]], np.int32)
    cache = B.KVCache(k, v, ks, vs, i32(pages.tolist()))
    rng = np.random.default_rng(46)
    x, tab, ws = bf16(rng, n, (n_q + 2 * n_kv) * hd), table(n, hd), workspace()
    Q, _ = B.fpt_rope_append(x.to(DEV), n_q, cache, torch.from_numpy(tab).to(DEV), i32([0]), cu_new=i32([0, n]), ws=ws)
    y = x.float().numpy().reshape(n, -1, hd)
    qk = OA.rope(y[:, :n_q + n_kv], tab, hd, False)
    local = np.array([[3, 1, 0, 2]], np.int32)                # the four pages on the host
    codes, scales = [np.zeros((4, n_kv, page, hd), np.int8) for _ in "kv"], [np.zeros((4, n_kv), np.float32) for _ in "kv"]
    OA.append(qk[:, n_q:], codes[0], scales[0], local[0], 0, page)
    OA.append(y[:, n_q + n_kv:], codes[1], scales[1], local[0], 0, page)
    for j, p in zip(local[0], pages[0]):
        assert np.array_equal(host(k[p]), codes[0][j]) and np.array_equal(host(v[p]), codes[1][j])
        assert np.array_equal(host(ks[p]), scales[0][j]) and np.array_equal(host(vs[p]), scales[1][j])
    K, V = B.fpt_kv_gather(cache, i32([0, n]), n, ws=ws)
    for got, j in ((K, 0), (V, 1)):
        want = OA.read(codes[j], scales[j], local[0], 0, n, page).reshape(n, -1)
        assert np.array_equal(bf16_host(got), torch.from_numpy(want).to(torch.bfloat16).float().numpy())
    last = Q[n - 1:n]
    o, lse = B.fpt_attn_decode(last, cache, i32([n]), want_lse=True, ws=ws)
    assert B.fpt_check_status(ws) == B.OK
    check_decode(o, lse, [n], local, codes, scales, last.cpu(), n_q, hd, page, hd ** -0.5)


def test_append_positions_and_pages_out_of_range_are_recorded():
    rng = np.random.default_rng(47)
    hd, page, n_q, n_kv = 64, 16, 2, 1
    tab = torch.from_numpy(table(50, hd)).to(DEV)
    x = bf16(rng, 6, (n_q + 2 * n_kv) * hd).to(DEV)
    for ctx, cu, spoil in (([45, 3], [0, 6, 6], None), ([-1, 3], [0, 3, 6], None), ([20, 3], [0, 3, 7], None), ([20, 3], [0, 4, 3], None),
                           ([20, 3], [0, 3, 6], -1), ([20, 3], [0, 3, 6], 1 << 20)):
        cache, pages, codes, scales = paged(rng, [30, 30], page, n_kv, hd)
        if spoil is not None:
            cache.pages[0, 1] = spoil
        ws = workspace()
        B.fpt_rope_append(x, n_q, cache, tab, i32(ctx), cu_new=i32(cu), ws=ws)
        assert B.fpt_check_status(ws) == B.ERR_INDEX, (ctx, cu, spoil)
        if spoil is not None:
            assert np.array_equal(host(cache.k)[pages[0]], codes[0][pages[0]])            # nothing went to another page
    cache, *_ = paged(rng, [30, 30], page, n_kv, hd)
    for first, cu in (([20, 20], [0, 13, 20]), ([-1, 0], [0, 5, 10]), ([0, 0], [0, 5, 999])):
        ws = workspace()
        B.fpt_kv_gather(cache, i32(cu), 20, first=i32(first), ws=ws)
        assert B.fpt_check_status(ws) == B.ERR_INDEX, (first, cu)


def test_calls_refuse_tensors_of_the_wrong_kind():
    rng = np.random.default_rng(48)
    cache, *_ = paged(rng, [20], 16, 2, 64)
    q, lens = bf16(rng, 1, 4 * 64).to(DEV), i32([20])
    for bad in (lambda: B.fpt_attn_decode(q.float(), cache, lens), lambda: B.fpt_attn_decode(q, cache, lens.long()),
                lambda: B.fpt_attn_decode(q, cache, lens.cpu()), lambda: B.fpt_attn_decode(q.cpu(), cache, lens),
                lambda: B.fpt_attn_decode(q, cache, i32([20, 20])), lambda: B.fpt_attn_decode(q[:, ::2], cache, lens),
                lambda: B.fpt_attn_decode(q, cache, lens, ws=torch.zeros(100, dtype=torch.uint8, device=DEV)),
                lambda: B.fpt_attn_decode(q.repeat(2, 1), cache, i32([20, 20])),          # a row more than the page table has
                lambda: B.fpt_attn_prompt(q, q[:, :128], q[:, :64], 4, 2, i32([0, 1])),
                lambda: B.fpt_kv_gather(cache, i32([0, 20]), 20, first=lens.long())):
        with pytest.raises(B.FptError):
            bad()


# ------------------------------------------------------------------------------------------------ few query rows, many keys
SPLIT = [
    # hd, n_q, n_kv, len_q, len_k (None: the same), causal
    (128, 32, 8, [64], [3000], True),
    (128, 4, 1, [1], [5000], True),
    (64, 24, 4, [100], [2777], True),
    (64, 8, 1, [33, 0, 70, 5], [1500, 900, 4000, 5], True),
    (128, 8, 2, [300], [2000], False),
    (128, 7, 1, [129, 3], [4000, 640], True),
    (64, 2, 2, [1700], None, True),                          # tasks of fewer tiles than the longest has parts
    (128, 2, 1, [600, 2], [100, 3333], True),                # rows that see nothing beside a long walk
    (128, 16, 1, [5] * 32, [2000 + 13 * i for i in range(32)], True),
    (64, 1, 1, [3], [20000], True),
]


@pytest.mark.parametrize("hd,n_q,n_kv,len_q,len_k,causal", SPLIT)
def test_prompt_keys_in_parts(hd, n_q, n_kv, len_q, len_k, causal):
    same, len_k = len_k is None, len_k or len_q
    rng = np.random.default_rng(sum(len_q) + hd + n_q + 1)
    q, k, v = prompt_case(rng, hd, n_q, n_kv, len_q, len_k)
    k[sum(len_k):] = math.nan
    v[sum(len_k):] = math.inf
    out = guarded_empty(q.shape, torch.bfloat16)
    out.fill_(7.0)
    room = B.fpt_workspace_bytes(B.OP_ATTN, 1, 1, 1)
    ws = torch.full((room + 4096,), 0x5A, dtype=torch.uint8, device=DEV)
    B.lib().fpt_reset_status(B._stream(), B._ptr(ws))
    _, lse = B.fpt_attn_prompt(q.to(DEV), k.to(DEV), v.to(DEV), n_q, n_kv, i32(offsets(len_q).tolist()),
                               cu_k=None if same else i32(offsets(len_k).tolist()), causal=causal, want_lse=True, O=out, ws=ws[:room])
    assert B.fpt_check_status(ws) == B.OK
    assert (ws[room:] == 0x5A).all()
    check_prompt(out, lse, q, k, v, n_q, n_kv, hd, len_q, len_k, causal)
    assert (bf16_host(out)[sum(len_q):] == 7).all()


@pytest.mark.parametrize("hd", [64, 128])
def test_prompt_parts_and_odd_values(hd):
    """Infinities and NaN in several parts' keys and values reach the queries that see them and no others."""
    rng = np.random.default_rng(51)
    n_q, n_kv, len_q, len_k = 4, 2, [100], [3000]
    q, k, v = prompt_case(rng, hd, n_q, n_kv, len_q, len_k, pad=0)
    v[2950, 3] = math.inf
    v[2990, 5] = math.nan
    v[1000, hd + 2] = math.nan                           # the second head, seen by every query
    k[2980, :hd] = math.nan
    o, lse = B.fpt_attn_prompt(q.to(DEV), k.to(DEV), v.to(DEV), n_q, n_kv, i32([0, 100]), cu_k=i32([0, 3000]), want_lse=True)
    args = [t.float().numpy().reshape(t.shape[0], -1, hd) for t in (q, k, v)]
    want, _, spread, mass = OA.attend(*args, hd ** -0.5, True)
    got = bf16_host(o).reshape(want.shape)
    fine = np.isfinite(want)
    assert fine.any() and not fine.all()
    assert (np.isfinite(got) == fine).all()
    assert (np.abs(got - want)[fine] <= out_bound(want, spread, mass, hd, HALF)[fine]).all()


def test_prompt_parts_captured_replayed_and_the_same_bits():
    """The sums of parts lie in the workspace: replays between other calls with it give the same bits."""
    rng = np.random.default_rng(52)
    hd, n_q, n_kv = 128, 8, 2
    q, k, v = (t.to(DEV) for t in prompt_case(rng, hd, n_q, n_kv, [90], [4000], pad=0))
    a, b, ws = i32([0, 90]), i32([0, 4000]), workspace()
    first, lse1 = B.fpt_attn_prompt(q, k, v, n_q, n_kv, a, cu_k=b, want_lse=True, ws=ws)
    out = torch.empty_like(first)
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        _, lse = B.fpt_attn_prompt(q, k, v, n_q, n_kv, a, cu_k=b, want_lse=True, O=out, ws=ws)
    page, lens = 64, [700, 9000]
    cache, pages, codes, scales, qd = decode_case(rng, hd, page, n_q, n_kv, lens)
    want, _ = B.fpt_attn_decode(qd.to(DEV), cache, i32(lens))
    for _ in range(4):
        out.fill_(0)
        lse.fill_(0)
        g.replay()
        o, _ = B.fpt_attn_decode(qd.to(DEV), cache, i32(lens), ws=ws)
        assert torch.equal(out.view(torch.int16), first.view(torch.int16)) and torch.equal(lse, lse1)
        assert torch.equal(o.view(torch.int16), want.view(torch.int16))
    assert B.fpt_check_status(ws) == B.OK


def test_calls_give_back_what_they_hold():
    """Outputs are freed with the caller's references, those of refused calls at once; arguments keep their counts."""
    import sys
    rng = np.random.default_rng(53)
    hd, page, n_q, n_kv = 64, 16, 4, 2
    cache, pages, codes, scales, q = decode_case(rng, hd, page, n_q, n_kv, [40])
    q, lens, ws = q.to(DEV), i32([40]), workspace()
    x, tab, cu = bf16(rng, 1, (n_q + 2 * n_kv) * hd).to(DEV), torch.from_numpy(table(64, hd)).to(DEV), i32([0, 1])
    kv = q[:, :n_kv * hd].contiguous()
    args = (q, lens, ws, x, tab, cu, kv, cache.k, cache.ref)

    def all_of_them():
        B.fpt_attn_decode(q, cache, lens, want_lse=True, ws=ws)
        B.fpt_attn_decode(q, cache, lens, O=kv.new_empty((1, n_q * hd)), ws=ws)
        B.fpt_rope_append(x, n_q, cache, tab, lens, want_k=True, ws=ws)
        B.fpt_kv_gather(cache, cu, 1, ws=ws)
        B.fpt_attn_prompt(q, kv, kv, n_q, n_kv, cu, want_lse=True, ws=ws)
        B.KVCache(cache.k, cache.v, cache.k_scale, cache.v_scale, cache.pages)
        for bad in (lambda: B.fpt_attn_decode(q, cache, lens, scale=-1.0, want_lse=True, ws=ws),
                    lambda: B.fpt_attn_decode(q, cache, lens, O=q[:, :64], ws=ws),
                    lambda: B.fpt_kv_gather(cache, cu, 1, V=q, ws=ws),
                    lambda: B.fpt_attn_prompt(q, kv, kv, n_q, n_kv, cu, scale=0.0, want_lse=True, ws=ws)):
            with pytest.raises(B.FptError):
                bad()
        with pytest.raises(TypeError):
            B.fpt_attn_decode(q, cache, lens, scale="one", ws=ws)

    B.set_allocator(None)                                # torch's own allocations are counted
    all_of_them()
    torch.cuda.synchronize()
    counts, held = [sys.getrefcount(a) for a in args], torch.cuda.memory_allocated()
    for _ in range(20):
        all_of_them()
    assert [sys.getrefcount(a) for a in args] == counts and torch.cuda.memory_allocated() == held


@pytest.mark.parametrize("hd,n_q,n_kv,n,most", [(128, 8, 2, 40, 300), (64, 1, 1, 100, 380), (128, 32, 2, 7, 65), (64, 12, 12, 33, 64), (128, 4, 4, 111, 700),
                                                   (128, 8, 2, 40, 190), (64, 1, 1, 100, 190)])
def test_decode_rows_kept_whole(hd, n_q, n_kv, n, most):
    """A CTA for each row, short rows: nothing is joined; sequences looked at 32 at a time, empty ones, one too long for its pages."""
    rng = np.random.default_rng(hd + n)
    lens = [int(x) for x in rng.integers(0, most + 1, n)]
    lens[0], lens[-1], lens[n // 2] = most, 1, 0
    cache, pages, codes, scales, q = decode_case(rng, hd, 32, n_q, n_kv, lens)
    ws = workspace()
    o, lse = B.fpt_attn_decode(q.to(DEV), cache, i32(lens), want_lse=True, ws=ws)
    assert B.fpt_check_status(ws) == B.OK
    check_decode(o, lse, lens, pages, codes, scales, q, n_q, hd, 32, hd ** -0.5)
    again = list(lens)
    again[1] = 1 << 29
    o2, _ = B.fpt_attn_decode(q.to(DEV), cache, i32(again), ws=ws)
    assert B.fpt_check_status(ws) == B.ERR_INDEX
    keep = [i for i in range(n) if i != 1]
    check_decode(o2[keep], None, [lens[i] for i in keep], pages[keep], codes, scales, q[keep], n_q, hd, 32, hd ** -0.5)


FEW_ROWS = [
    # hd, page, n_q, n_kv, rot, interleaved, new, ctx: less than two rows a sequence
    (128, 64, 8, 2, 128, 0, [1] * 20 + [0] * 5 + [9, 2], [(37 * i) % 130 for i in range(25)] + [60, 63]),
    (64, 16, 4, 4, 64, 1, [0] * 7 + [40] + [0] * 30 + [1, 3], [5] * 7 + [10] + [0] * 30 + [15, 14]),
    (128, 128, 2, 1, 64, 0, [2, 0, 1, 0, 0, 2], [127, 3, 128, 0, 9, 126]),
]


@pytest.mark.parametrize("hd,page,n_q,n_kv,rot,inter,new,ctx", FEW_ROWS)
def test_append_of_few_rows_a_sequence(hd, page, n_q, n_kv, rot, inter, new, ctx):
    test_append_matches_the_oracle_bit_for_bit(hd, page, n_q, n_kv, rot, inter, new, ctx, False)


def test_few_rows_turned_without_a_cache_and_offsets_out_of_range():
    rng = np.random.default_rng(54)
    hd, n_q, n_kv, new = 64, 4, 2, [0, 2, 1, 0, 1, 3]
    rows, ctx = sum(new), [3, 9, 0, 4, 63, 64]
    x, tab, ws = bf16(rng, rows, (n_q + 2 * n_kv) * hd), table(70, hd), workspace()
    tabd, cu = torch.from_numpy(tab).to(DEV), offsets(new)
    q, k = B.fpt_rope_append(x.to(DEV), n_q, B.KVCache.heads(n_kv, hd), tabd, i32(ctx), cu_new=i32(cu.tolist()), want_k=True, ws=ws)
    assert B.fpt_check_status(ws) == B.OK
    at = np.concatenate([np.arange(c, c + n) for c, n in zip(ctx, new)])
    want = OA.rope(x.float().numpy().reshape(rows, -1, hd)[:, :n_q + n_kv], tab[at], hd, False)
    assert np.array_equal(bf16_host(q), want[:, :n_q].reshape(rows, -1)) and np.array_equal(bf16_host(k), want[:, n_q:].reshape(rows, -1))
    for bad in ([9, 9, 9, 9, 9, 9, 12], [0, 2, 3, 3, 4, 7, 8], [-1, 0, 0, 0, 0, 0, 0], [0, 3, 1, 1, 1, 1, 1]):
        ws = workspace()
        B.fpt_rope_append(x.to(DEV), n_q, B.KVCache.heads(n_kv, hd), tabd, i32(ctx), cu_new=i32(bad), ws=ws)
        assert B.fpt_check_status(ws) == B.ERR_INDEX, bad


PADDED = [
    # hd, n_q, n_kv, len_q, len_k (None: the same), causal: groups that no power of two divides, short sequences
    (128, 40, 8, [9, 6, 1, 14, 0, 11], None, True),
    (64, 20, 4, [78, 19, 51], [90, 19, 333], True),
    (128, 14, 2, [1, 1, 1], [700, 3, 130], True),
    (64, 36, 3, [13, 16, 2], None, True),
    (128, 19, 1, [7, 5], [64, 200], False),
    (64, 3, 1, [1], [9000], True),                           # one head of padding, keys in parts
    (128, 10, 2, [12], [3000], True),
]


@pytest.mark.parametrize("hd,n_q,n_kv,len_q,len_k,causal", PADDED)
def test_prompt_heads_that_fill_no_tile(hd, n_q, n_kv, len_q, len_k, causal):
    test_prompt(hd, n_q, n_kv, len_q, len_k, causal)


UNEVEN = [
    # hd, n_q, n_kv, len_q, len_k (None: the same), causal: only the tasks with many keys are split
    (64, 2, 2, [3000], None, True),
    (128, 5, 1, [2900, 10], None, True),
    (128, 4, 2, [900, 100, 700], [900, 2500, 1400], True),
    (64, 8, 2, [64, 1, 300], [100, 6000, 3000], False),
    (128, 16, 2, [400], [1500], True),
]


@pytest.mark.parametrize("hd,n_q,n_kv,len_q,len_k,causal", UNEVEN)
def test_prompt_tasks_of_uneven_length(hd, n_q, n_kv, len_q, len_k, causal):
    test_prompt_keys_in_parts(hd, n_q, n_kv, len_q, len_k, causal)
