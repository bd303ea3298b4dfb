"""The attention calls at the edges of what they allow: batches without a row or a key, offsets that do not ascend, codes of errors beside
one another, what a program does between calls."""
import math

import numpy as np
import pytest
import torch

from oracle import attention as OA
from paper_2506_04985_b200 import binding as B
from helpers import DEV, bf16_host, guarded_empty, host
from test_gpu_attn import bf16, check_decode, check_prompt, decode_case, i32, offsets, paged, prompt_case, table, workspace

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("n,rows", [(3, 1000), (41, 1000), (300, 2000), (300, 400)])
def test_offsets_that_do_not_ascend_stay_inside_the_buffers(n, rows):
    """Sequences that are fine by themselves claim the same tasks, from one warp and from several; outputs end with their guard bands, rows of
    the cache's pages that no sequence has stay as they were."""
    rng = np.random.default_rng(n)
    hd, page, n_q, n_kv = 64, 16, 2, 1
    cu = [0, rows] + [5 + i * (rows - 90) // n for i in range(n - 2)] + [rows]
    cache, pages, codes, scales = paged(rng, [max(b - a, 0) + page for a, b in zip(cu, cu[1:])], page, n_kv, hd)
    x, tab = bf16(rng, rows, (n_q + 2 * n_kv) * hd).to(DEV), torch.from_numpy(table(rows + 64, hd)).to(DEV)
    for _ in range(3):
        ws = workspace()
        ctx = i32([int(c) for c in rng.integers(0, page, n)])
        Q, K = guarded_empty((rows, n_q * hd), torch.bfloat16), guarded_empty((rows, n_kv * hd), torch.bfloat16)
        B.fpt_rope_append(x, n_q, cache, tab, ctx, cu_new=i32(cu), Q=Q, K=K, ws=ws)
        assert B.fpt_check_status(ws) == B.ERR_INDEX
        ws = workspace()
        K, V = guarded_empty((rows, n_kv * hd), torch.bfloat16), guarded_empty((rows, n_kv * hd), torch.bfloat16)
        B.fpt_kv_gather(cache, i32(cu), rows, first=ctx, K=K, V=V, ws=ws)
        assert B.fpt_check_status(ws) == B.ERR_INDEX
    free = sorted(set(range(cache.k.shape[0])) - {int(p) for p in pages.ravel() if p >= 0})
    assert len(free) == 2 and np.array_equal(host(cache.k)[free], codes[0][free]) and np.array_equal(host(cache.v_scale)[free], scales[1][free])


def test_an_index_out_of_range_covers_no_wait_that_gave_up():
    """Both kinds of error on one workspace, in either order: the one that spoils every output is the one that is reported."""
    rng = np.random.default_rng(2)
    cache, _, _, _, q = decode_case(rng, 64, 16, 2, 1, [20])
    q, too_long = q.to(DEV), i32([1 << 20])
    for order in (0, 1):
        ws = workspace()
        for what in ("index", "wait") if order == 0 else ("wait", "index"):
            if what == "index":
                B.fpt_attn_decode(q, cache, too_long, ws=ws)
                assert B.fpt_check_status(ws) == (B.ERR_INDEX if order == 0 else B.ERR_TIMEOUT)
            else:
                B.fpt_selftest_wait_timeout(ws, limit_us=2000)
                assert B.fpt_check_status(ws) == B.ERR_TIMEOUT
        assert B.lib().fpt_reset_status(B._stream(), B._ptr(ws)) == B.OK
        assert B.fpt_check_status(ws) == B.OK
        B.fpt_attn_decode(q, cache, too_long, ws=ws)
        assert B.fpt_check_status(ws) == B.ERR_INDEX


def test_a_page_table_that_grows_between_calls():
    """A server's way: the table and the storage of a cache are replaced as contexts grow; the old ones' memory goes to others."""
    rng = np.random.default_rng(3)
    hd, page, n_q, n_kv = 64, 16, 4, 2
    cache, pages, codes, scales, q = decode_case(rng, hd, page, n_q, n_kv, [60, 9])
    q, ws = q.to(DEV), workspace()
    whole, table_2 = pages.copy(), torch.from_numpy(pages[:1, :2].copy()).to(DEV)
    cache.pages = table_2
    o, _ = B.fpt_attn_decode(q[:1], cache, i32([30]), ws=ws)
    check_decode(o, None, [30], pages, codes, scales, q.cpu(), n_q, hd, page, hd ** -0.5)
    with pytest.raises(B.FptError):                        # a row that this table has not
        B.fpt_attn_decode(q, cache, i32([30, 9]), ws=ws)
    cache.pages = i32(whole.tolist())
    del table_2
    spoil = [torch.full((1, 2), 1 << 29, dtype=torch.int32, device=DEV) for _ in range(8)]
    for name in ("k", "v", "k_scale", "v_scale"):
        setattr(cache, name, getattr(cache, name).clone())
    o, _ = B.fpt_attn_decode(q, cache, i32([60, 9]), ws=ws)
    assert B.fpt_check_status(ws) == B.OK and len(spoil) == 8
    check_decode(o, None, [60, 9], pages, codes, scales, q.cpu(), n_q, hd, page, hd ** -0.5)
    x, tab = bf16(rng, 1, (n_q + 2 * n_kv) * hd).to(DEV), torch.from_numpy(table(70, hd)).to(DEV)
    keep = cache.pages
    for bad in (keep.long(), keep.cpu(), keep[:, ::2], None):
        cache.pages = bad
        for call in (lambda: B.fpt_attn_decode(q, cache, i32([60, 9])), lambda: B.fpt_kv_gather(cache, i32([0, 5]), 5),
                     lambda: B.fpt_rope_append(x, n_q, cache, tab, i32([60]))):
            with pytest.raises(B.FptError) as e:
                call()
            assert e.value.code == B.ERR_BAD_ARG


def test_read_back_of_nothing():
    """Prefixes that are all empty, a single one among them; into tensors of the caller's; an offset beyond is recorded as ever."""
    rng = np.random.default_rng(4)
    cache, *_ = paged(rng, [0, 0, 5], 16, 2, 64)
    for n in (1, 3):
        ws = workspace()
        K, V = B.fpt_kv_gather(cache, i32([0] * (n + 1)), 0, ws=ws)
        assert K.shape == V.shape == (0, 128) and K.dtype == torch.bfloat16 and B.fpt_check_status(ws) == B.OK
        wide = guarded_empty((4, 256), torch.bfloat16)
        B.fpt_kv_gather(cache, i32([0] * (n + 1)), 0, K=wide[:0, :128], V=wide[:0, 128:], first=i32([3] * n), ws=ws)
        assert B.fpt_check_status(ws) == B.OK
        B.fpt_kv_gather(cache, i32([0] * n + [5]), 0, ws=ws)
        assert B.fpt_check_status(ws) == B.ERR_INDEX


@pytest.mark.parametrize("hd,n_q,n_kv,lens", [(128, 4, 2, [5, 0, 300]), (64, 5, 1, [1]), (64, 2, 2, [3] * 150), (128, 32, 8, [17] * 40)])
@pytest.mark.parametrize("causal", [True, False])
def test_prompt_without_any_key(hd, n_q, n_kv, lens, causal):
    rng = np.random.default_rng(5)
    q = bf16(rng, sum(lens) + 2, n_q * hd)
    q[0] = math.nan
    out, ws = guarded_empty(q.shape, torch.bfloat16), workspace()
    out.fill_(7.0)
    none = torch.empty((0, n_kv * hd), dtype=torch.bfloat16, device=DEV)
    _, lse = B.fpt_attn_prompt(q.to(DEV), none, none, n_q, n_kv, i32(offsets(lens).tolist()), cu_k=i32([0] * (len(lens) + 1)), causal=causal,
                               want_lse=True, O=out, ws=ws)
    assert B.fpt_check_status(ws) == B.OK
    rows = sum(lens)
    assert (bf16_host(out)[:rows] == 0).all() and (bf16_host(out)[rows:] == 7).all() and np.isneginf(host(lse)[:rows]).all()
    B.fpt_attn_prompt(q.to(DEV), none, none, n_q, n_kv, i32(offsets(lens).tolist()), cu_k=i32([0] * len(lens) + [1]), O=out, ws=ws)
    assert B.fpt_check_status(ws) == B.ERR_INDEX


@pytest.mark.parametrize("n", [20, 100, 129, 200, 5000])
@pytest.mark.parametrize("what", ["queries", "keys", "queries, far", "keys of no query"])
def test_prompt_offsets_that_do_not_ascend_are_recorded(n, what):
    """Wherever it stands, and whether or not a task of the spoilt sequence would be looked for."""
    rng = np.random.default_rng(n)
    hd, n_q, n_kv, lens = 64, 2, 1, [4] * n
    q, k, v = (t.to(DEV) for t in prompt_case(rng, hd, n_q, n_kv, lens, lens, pad=0))
    for at in (3, n // 2, n - 2):
        a, b = offsets(lens), offsets(lens)
        if what == "keys of no query":
            a[at:] -= 4
        off = b if what.startswith("keys") else a
        off[at] = 0 if what.endswith("far") else off[at - 1] - 2
        ws, out = workspace(), guarded_empty(q.shape, torch.bfloat16)
        B.fpt_attn_prompt(q, k, v, n_q, n_kv, i32(a.tolist()), cu_k=i32(b.tolist()), O=out, ws=ws)
        assert B.fpt_check_status(ws) == B.ERR_INDEX, at
        ws = workspace()
        B.fpt_attn_prompt(q, k, v, n_q, n_kv, i32(offsets(lens).tolist()), cu_k=i32(offsets(lens).tolist()), O=out, ws=ws)
        assert B.fpt_check_status(ws) == B.OK


@pytest.mark.parametrize("hd", [64, 128])
def test_prompt_infinities_keep_their_sign_and_nan_their_place(hd):
    rng = np.random.default_rng(23)
    n_q, n_kv, lens = 4, 2, [200, 70, 30]
    q, k, v = prompt_case(rng, hd, n_q, n_kv, lens, lens, pad=0)
    v[150, 3] = math.inf
    v[190, 3] = -math.inf
    v[20, 5] = -math.inf
    v[199, hd + 1] = math.nan
    k[180, hd:] = math.nan
    v[260, :] = math.nan
    k[205, 0] = math.inf
    o, lse = B.fpt_attn_prompt(q.to(DEV), k.to(DEV), v.to(DEV), n_q, n_kv, i32(offsets(lens).tolist()), want_lse=True)
    check_prompt(o, lse, q, k, v, n_q, n_kv, hd, lens, lens, True)


@pytest.mark.parametrize("hd", [64, 128])
def test_prompt_parts_keep_infinities_and_nan_apart(hd):
    rng = np.random.default_rng(51)
    n_q, n_kv, len_q, len_k = 4, 2, [100], [3000]
    q, k, v = prompt_case(rng, hd, n_q, n_kv, len_q, len_k, pad=0)
    v[2950, 3] = math.inf
    v[2960, 4] = -math.inf
    v[2990, 5] = math.nan
    v[500, 7] = -math.inf
    v[1000, hd + 2] = math.nan
    k[2980, :hd] = math.nan
    o, lse = B.fpt_attn_prompt(q.to(DEV), k.to(DEV), v.to(DEV), n_q, n_kv, i32([0, 100]), cu_k=i32([0, 3000]), want_lse=True)
    check_prompt(o, lse, q, k, v, n_q, n_kv, hd, len_q, len_k, True)


@pytest.mark.parametrize("hd,n_q,n_kv,lens,pre", [
    (128, 8, 2, [33, 200, 5], [0, 100, 700]), (64, 10, 2, [3, 9, 0, 4], [5, 5, 5, 5]), (64, 2, 1, [3] * 150, [7] * 150), (128, 4, 1, [16], [4000])])
def test_prompt_that_begins_behind_the_first_row(hd, n_q, n_kv, lens, pre):
    rng = np.random.default_rng(5)
    len_k = [a + b for a, b in zip(lens, pre)]
    q, k, v = prompt_case(rng, hd, n_q, n_kv, lens, len_k, pad=9)
    at_q, at_k = 5, 7
    Q, K, V = (torch.cat([torch.full((n, t.shape[1]), math.nan, dtype=t.dtype), t]) for t, n in ((q, at_q), (k, at_k), (v, at_k)))
    out, ws = guarded_empty(Q.shape, torch.bfloat16), workspace()
    out.fill_(7.0)
    _, lse = B.fpt_attn_prompt(Q.to(DEV), K.to(DEV), V.to(DEV), n_q, n_kv, i32((offsets(lens) + at_q).tolist()),
                               cu_k=i32((offsets(len_k) + at_k).tolist()), want_lse=True, O=out, ws=ws)
    assert B.fpt_check_status(ws) == B.OK
    check_prompt(out[at_q:], lse[at_q:], q, k, v, n_q, n_kv, hd, lens, len_k, True)
    assert (bf16_host(out)[:at_q] == 7).all() and (bf16_host(out)[at_q + sum(lens):] == 7).all()


@pytest.mark.parametrize("new,ctx", [([70, 1, 30], [5, 63, 40]), ([1, 0, 2, 1, 0], [63, 5, 64, 127, 9])])
def test_append_and_read_back_that_begin_behind_the_first_row(new, ctx):
    rng = np.random.default_rng(6)
    hd, page, n_q, n_kv, at = 64, 64, 4, 2, 6
    cache, pages, codes, scales = paged(rng, [a + b for a, b in zip(new, ctx)], page, n_kv, hd)
    rows = sum(new)
    x = bf16(rng, rows + at + 3, (n_q + 2 * n_kv) * hd)
    tab, ws, cu = table(300, hd), workspace(), offsets(new) + at
    Q = guarded_empty((rows + at + 3, n_q * hd), torch.bfloat16)
    Q.fill_(7.0)
    B.fpt_rope_append(x.to(DEV), n_q, cache, torch.from_numpy(tab).to(DEV), i32(ctx), cu_new=i32(cu.tolist()), Q=Q, ws=ws)
    y = x.float().numpy().reshape(-1, n_q + 2 * n_kv, hd)
    for i, (n, c) in enumerate(zip(new, ctx)):
        if n:
            qk = OA.rope(y[cu[i]:cu[i + 1], :n_q + n_kv], tab[c:c + n], hd, False)
            assert np.array_equal(bf16_host(Q)[cu[i]:cu[i + 1]].reshape(n, n_q, hd), qk[:, :n_q])
            OA.append(qk[:, n_q:], codes[0], scales[0], pages[i], c, page)
            OA.append(y[cu[i]:cu[i + 1], n_q + n_kv:], codes[1], scales[1], pages[i], c, page)
    assert (bf16_host(Q)[:at] == 7).all() and (bf16_host(Q)[at + rows:] == 7).all()
    for got, want in zip((cache.k_scale, cache.v_scale, cache.k, cache.v), (*scales, *codes)):
        assert np.array_equal(host(got), want)
    ends = [a + b for a, b in zip(new, ctx)]
    K, V = (guarded_empty((sum(ends) + at + 2, n_kv * hd), torch.bfloat16) for _ in "kv")
    K.fill_(7.0), V.fill_(7.0)
    co = offsets(ends) + at
    B.fpt_kv_gather(cache, i32(co.tolist()), K.shape[0], K=K, V=V, ws=ws)
    assert B.fpt_check_status(ws) == B.OK
    for i, e in enumerate(ends):
        for got, j in ((K, 0), (V, 1)):
            want = torch.from_numpy(OA.read(codes[j], scales[j], pages[i], 0, e, page)).to(torch.bfloat16).float().numpy().reshape(e, -1)
            assert np.array_equal(bf16_host(got)[co[i]:co[i + 1]], want)
    assert (bf16_host(K)[:at] == 7).all() and (bf16_host(K)[-2:] == 7).all()


@pytest.mark.parametrize("hd,n_q,n_kv", [(128, 8, 2), (64, 32, 2)])
def test_decode_value_scales_far_apart(hd, n_q, n_kv):
    """Pages whose values lie 2^109 apart beside one another, those below 2^-80 that count as zeros, and a page of zeros: the sums of
    weights do not feel the scales."""
    rng = np.random.default_rng(6)
    page, lens = 16, [500, 40, 70]
    cache, pages, codes, scales, q = decode_case(rng, hd, page, n_q, n_kv, lens)
    for p, at in enumerate(pages[0]):
        if at >= 0:
            scales[1][at] = 2.0 ** (30, -79, 0, -3)[p % 4]
    zero = pages[1][0]
    scales[1][zero], codes[1][zero] = 0, 0
    scales[1][pages[1][1:3]] = 2.0 ** 30
    scales[1][pages[2][:5]] = 2.0 ** -79
    cache.v_scale.copy_(torch.from_numpy(scales[1])), cache.v.copy_(torch.from_numpy(codes[1]))
    o, lse = B.fpt_attn_decode(q.to(DEV), cache, i32(lens), want_lse=True)
    check_decode(o, lse, lens, pages, codes, scales, q, n_q, hd, page, hd ** -0.5)


@pytest.mark.parametrize("hd,n_q,n_kv,lens", [(64, 1, 1, [60000]), (128, 4, 1, [45000]), (64, 16, 1, [33000]), (128, 20, 1, [40000, 3])])
def test_decode_one_row_over_every_cta(hd, n_q, n_kv, lens):
    """A row in more parts than the join looks at in a step, or has room for weights of."""
    rng = np.random.default_rng(7)
    cache, pages, codes, scales, q = decode_case(rng, hd, 64, n_q, n_kv, lens)
    ws = workspace()
    o, lse = B.fpt_attn_decode(q.to(DEV), cache, i32(lens), want_lse=True, ws=ws)
    assert B.fpt_check_status(ws) == B.OK
    check_decode(o, lse, lens, pages, codes, scales, q, n_q, hd, 64, hd ** -0.5)
