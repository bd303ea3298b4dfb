"""The attention between the library's two attention projections, as work to be timed: rotary positions with the append
to a paged 8-bit cache, reading cached tokens back in 16 bits, attention of single tokens over the cache, causal attention
of whole prompts.

`own` false: elementary torch operations in float32.  `own` true: the calls of the library's entry points on the same
inputs.  `exact` restates each definition in 64 bits; where an operator defines a rounding (bf16 keys before they are
coded, the codes themselves), it rounds there too.

What a program holds before a call: the projections' output, the table of rotations, a page table, the cache, a cleared
workspace, lengths and offsets on the device.  Lengths follow from the case alone, so that `work` knows them.
"""
import math
import random

import torch

own = False
DEV = "cuda"
WORKSPACE_BYTES = 16 << 20


# ------------------------------------------------------------------------------------------------ cases
def listed():
    def case(name, kind, n_q=32, n_kv=8, hd=128, page=64, **more):
        return dict(name=name, kind=kind, n_q=n_q, n_kv=n_kv, hd=hd, page=page, **more)

    return [
        # a decode step of 64 users: each adds one token to a page it shares with earlier ones
        case("append_decode_64", "append", n_seqs=64, new_lo=1, new_hi=1, ctx_lo=1, ctx_hi=4000, rot=128, layout="half", shape=1),
        # packed prompts of several users behind prefixes that end inside a page; half of the head rotated, in pairs
        case("append_prompts_8192", "append", n_seqs=7, new_lo=700, new_hi=1640, ctx_lo=0, ctx_hi=300, rot=64,
             layout="pairs", shape=2),
        # the cached prefix of one long prompt in 16 bits again, for the attention of its next chunk
        case("gather_32768", "gather", n_seqs=1, len_lo=32768, len_hi=32768, shape=3),
        # short ragged prefixes in small pages, 64-value heads
        case("gather_ragged_37", "gather", n_q=16, n_kv=16, hd=64, page=16, n_seqs=37, len_lo=1, len_hi=1000, shape=4),
        # one user, short context: the cost of a call
        case("decode_1x1000", "decode", n_seqs=1, len_lo=1000, len_hi=1000, shape=5),
        # one user, very long context: the work of one sequence over the whole GPU
        case("decode_1x131071", "decode", n_seqs=1, len_lo=131071, len_hi=131071, shape=6),
        # a full batch of ragged contexts, heads of the 70B-class model
        case("decode_64_ragged", "decode", n_q=64, n_seqs=64, len_lo=17, len_hi=12000, shape=7),
        # a small batch with an empty slot, a query head for each key head, 64-value heads, pages of 16 tokens
        case("decode_9_heads64", "decode", n_q=12, n_kv=12, hd=64, page=16, n_seqs=9, len_lo=0, len_hi=2500, shape=8),
        # many short prompts packed together
        case("prompt_33_short", "prompt", n_seqs=33, q_lo=1, q_hi=300, pre_lo=0, pre_hi=0, shape=9),
        # the headline token count as one prompt
        case("prompt_2048", "prompt", n_seqs=1, q_lo=2048, q_hi=2048, pre_lo=0, pre_hi=0, shape=10),
        # a long prompt
        case("prompt_8192", "prompt", n_seqs=1, q_lo=8192, q_hi=8192, pre_lo=0, pre_hi=0, shape=11),
        # chunks of four prompts behind their prefixes, 64-value heads
        case("prompt_chunks_4", "prompt", n_q=24, n_kv=4, hd=64, n_seqs=4, q_lo=333, q_hi=777, pre_lo=500, pre_hi=7000, shape=12),
    ]


def draw(rng):
    def near(lo, hi):                                   # spread over the logarithm
        return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))

    kind = rng.choice(["append", "gather", "decode", "decode", "prompt", "prompt"])
    hd = rng.choice([64, 128, 128])
    n_kv = rng.choice([1, 2, 4, 8, 8, 12])
    group = rng.choice([1, 2, 4, 4, 5, 7, 8, 16])
    group = min(group, 64 // n_kv)
    c = dict(kind=kind, n_q=n_kv * group, n_kv=n_kv, hd=hd, page=rng.choice([16, 32, 64, 64, 128]),
             n_seqs=near(1, 64), shape=rng.randrange(1 << 20))
    if kind == "append":
        new = 1 if rng.random() < 0.4 else near(2, max(2, 8192 // c["n_seqs"]))
        c.update(new_lo=max(1, new // 3), new_hi=new, ctx_lo=0, ctx_hi=near(1, 2000),
                 rot=rng.choice([hd, hd, hd // 2]), layout=rng.choice(["half", "half", "pairs"]))
    elif kind == "gather":
        hi = near(1, 32768 // c["n_seqs"])
        c.update(len_lo=rng.randint(0, hi), len_hi=hi)
    elif kind == "decode":
        hi = min(near(1, 131072), 360_000_000 // (c["n_seqs"] * n_kv * hd))
        c.update(len_lo=rng.randint(0, hi), len_hi=hi)
    else:
        pre = 0 if rng.random() < 0.6 else near(1, 4096)
        most = 2 ** 31 // (c["n_seqs"] * c["n_q"])      # query heads times queries times keys: as many as the longest listed prompt
        hi = near(1, max(1, min(8192, int(math.sqrt(most + pre * pre / 4) - pre / 2))))
        c.update(q_lo=max(1, hi // 4), q_hi=hi, pre_lo=0, pre_hi=pre)
    return c


def _lengths(case):
    """The lengths of a case's sequences: {name: [n_seqs]}; they follow from the case alone."""
    rng = random.Random(case["shape"])
    n = case["n_seqs"]

    def some(lo, hi):
        return [rng.randint(case[lo], case[hi]) for _ in range(n)]

    if case["kind"] == "append":
        return dict(new=some("new_lo", "new_hi"), ctx=some("ctx_lo", "ctx_hi"))
    if case["kind"] == "prompt":
        q, pre = some("q_lo", "q_hi"), some("pre_lo", "pre_hi")
        return dict(q=q, k=[a + b for a, b in zip(q, pre)])
    lens = some("len_lo", "len_hi")
    if case["kind"] == "decode" and n > 4 and case["len_lo"] == 0:
        lens[n // 2] = 0
    return dict(len=lens)


def work(case):
    n_q, n_kv, hd, page, L = case["n_q"], case["n_kv"], case["hd"], case["page"], _lengths(case)

    def pages(n):
        return -(-n // page)

    if case["kind"] == "append":
        t = sum(L["new"])
        back = sum(c % page + n for c, n in zip(L["ctx"], L["new"]))             # tokens of the pages that change
        blocks = sum(pages(c % page + n) for c, n in zip(L["ctx"], L["new"]))
        # rows in, rotated queries and keys out, codes out; the changed pages' codes in and their values out; scales
        b = t * (n_q + 2 * n_kv) * hd * 2 + t * (n_q + n_kv) * hd * 2 + t * 2 * n_kv * hd
        b += t * case["rot"] * 4 + back * 2 * n_kv * hd * 3 + blocks * 2 * n_kv * 8
        return dict(bytes=b, flops=t * ((n_q + n_kv) * case["rot"] * 3 + 2 * n_kv * hd * 3) + back * 2 * n_kv * hd)
    if case["kind"] == "gather":
        t = sum(L["len"])
        return dict(bytes=t * 2 * n_kv * hd * 3 + sum(map(pages, L["len"])) * 2 * n_kv * 4, flops=t * 2 * n_kv * hd)
    if case["kind"] == "decode":
        t = sum(L["len"])
        b = t * 2 * n_kv * hd + sum(map(pages, L["len"])) * (2 * n_kv * 4 + 4) + len(L["len"]) * n_q * (hd * 4 + 4)
        return dict(bytes=b, flops=t * n_q * hd * 4)
    seen = sum(q * (k - q) + q * (q + 1) // 2 for q, k in zip(L["q"], L["k"]))
    b = sum(L["q"]) * n_q * (hd * 4 + 4) + sum(L["k"]) * n_kv * hd * 4
    return dict(bytes=b, flops=seen * n_q * hd * 4)


# ------------------------------------------------------------------------------------------------ inputs
def _gen(seed):
    g = torch.Generator(device=DEV)
    g.manual_seed(seed)
    return g


def _dev_i32(v):
    return torch.tensor(v, dtype=torch.int32, device=DEV)


def _offsets(v):
    return _dev_i32([sum(v[:i]) for i in range(len(v) + 1)])


def _projected(g, rows, n_q, n_kv, hd):
    """Rows as the fused projection leaves them: queries, keys with a few large channels, values."""
    x = torch.randn((rows, n_q + 2 * n_kv, hd), generator=g, device=DEV, dtype=torch.float32)
    gain = 1.0 + 7.0 * (torch.rand((n_kv, hd), generator=g, device=DEV) < 0.03).float()
    x[:, n_q:n_q + n_kv] *= gain
    return x.to(torch.bfloat16).view(rows, (n_q + 2 * n_kv) * hd)


def _rotations(n_pos, rot):
    """cos and sin of position * frequency, base 500000 as long-context models take it."""
    f = 500000.0 ** (-torch.arange(0, rot, 2, device=DEV, dtype=torch.float64) / rot)
    a = torch.arange(n_pos, device=DEV, dtype=torch.float64)[:, None] * f
    return torch.stack([a.cos(), a.sin()], -1).float()


def _cache(g, n_kv, hd, page, lens):
    """A cache whose pages hold the sequences' tokens in an order of their own, with a few pages to spare."""
    need = [-(-n // page) for n in lens]
    n_pages = sum(need) + 3
    order = torch.randperm(n_pages, generator=g, device=DEV).to(torch.int32)
    width = max(max(need), 1)
    at = torch.arange(width, device=DEV)[None, :] + _offsets(need)[:-1, None].long()
    pages = torch.where(torch.arange(width, device=DEV)[None, :] < _dev_i32(need)[:, None], order[at.clamp(max=n_pages - 1)], 0)
    shape = (n_pages, n_kv, page, hd)
    k = torch.randint(-127, 128, shape, generator=g, device=DEV, dtype=torch.int8)
    v = torch.randint(-127, 128, shape, generator=g, device=DEV, dtype=torch.int8)
    k_scale = (1.5 + 2.0 * torch.rand((n_pages, n_kv), generator=g, device=DEV)) / 127
    v_scale = (1.5 + 2.0 * torch.rand((n_pages, n_kv), generator=g, device=DEV)) / 127
    return dict(k=k, v=v, k_scale=k_scale, v_scale=v_scale, pages=pages.to(torch.int32).contiguous())


def prepare(case, seed):
    g = _gen(seed)
    n_q, n_kv, hd, page, L = case["n_q"], case["n_kv"], case["hd"], case["page"], _lengths(case)
    s = dict(case=case, ws=torch.zeros(WORKSPACE_BYTES, dtype=torch.uint8, device=DEV))
    if case["kind"] == "append":
        end = [c + n for c, n in zip(L["ctx"], L["new"])]
        first = [c // page * page for c in L["ctx"]]
        s.update(_cache(g, n_kv, hd, page, end), qkv=_projected(g, sum(L["new"]), n_q, n_kv, hd),
                 table=_rotations(max(end), case["rot"]), cu_new=_offsets(L["new"]), ctx=_dev_i32(L["ctx"]),
                 first=_dev_i32(first), cu_back=_offsets([e - f for e, f in zip(end, first)]),
                 n_back=sum(end) - sum(first))
    elif case["kind"] == "gather":
        s.update(_cache(g, n_kv, hd, page, L["len"]), cu=_offsets(L["len"]), total=sum(L["len"]))
    elif case["kind"] == "decode":
        s.update(_cache(g, n_kv, hd, page, L["len"]), lens=_dev_i32(L["len"]))
        s["q"] = torch.randn((case["n_seqs"], n_q * hd), generator=g, device=DEV).to(torch.bfloat16)
    else:
        tq, tk = sum(L["q"]), sum(L["k"])
        kv = _projected(g, tk, 0, n_kv, hd)
        s.update(q=torch.randn((tq, n_q * hd), generator=g, device=DEV).to(torch.bfloat16),
                 k=kv[:, :n_kv * hd], v=kv[:, n_kv * hd:], cu_q=_offsets(L["q"]), cu_k=_offsets(L["k"]),
                 max_q=max(L["q"]), max_k=max(L["k"]))
    return s


# ------------------------------------------------------------------------------------------------ one pass
def run(s):
    case = s["case"]
    if own:
        return _own[case["kind"]](s)
    return _plain[case["kind"]](s)


def _handle(s):
    from paper_2506_04985_b200 import binding as B
    return B, B.KVCache(s["k"], s["v"], s["k_scale"], s["v_scale"], s["pages"])


def _own_append(s):
    B, cache = _handle(s)
    c = s["case"]
    q, k = B.fpt_rope_append(s["qkv"], c["n_q"], cache, s["table"], s["ctx"], cu_new=s["cu_new"], ws=s["ws"],
                             layout=B.ROPE_HALF if c["layout"] == "half" else B.ROPE_INTERLEAVED, want_k=True)
    kb, vb = B.fpt_kv_gather(cache, s["cu_back"], s["n_back"], first=s["first"], ws=s["ws"])
    return dict(q=q, k=k, cached_k=kb, cached_v=vb, k_scale=cache.k_scale, v_scale=cache.v_scale)


def _own_gather(s):
    B, cache = _handle(s)
    k, v = B.fpt_kv_gather(cache, s["cu"], s["total"], ws=s["ws"])
    return dict(k=k, v=v)


def _own_decode(s):
    B, cache = _handle(s)
    o, lse = B.fpt_attn_decode(s["q"], cache, s["lens"], want_lse=True, ws=s["ws"])
    return dict(o=o, lse=lse)


def _own_prompt(s):
    from paper_2506_04985_b200 import binding as B
    c = s["case"]
    o, lse = B.fpt_attn_prompt(s["q"], s["k"], s["v"], c["n_q"], c["n_kv"], s["cu_q"], cu_k=s["cu_k"], want_lse=True,
                               ws=s["ws"])
    return dict(o=o, lse=lse)


_own = dict(append=_own_append, gather=_own_gather, decode=_own_decode, prompt=_own_prompt)


# ------------------------------------------------------------------------------------------------ the plain forms
def _rows(cu, total):
    """For packed rows: the sequence of each and its place in it."""
    n = cu.numel() - 1
    seq = torch.repeat_interleave(torch.arange(n, device=DEV), (cu[1:] - cu[:-1]).long(), output_size=total)
    return seq, torch.arange(total, device=DEV) - cu[seq].long()


def _rotate(x, cs, sn, rot, layout):
    """x [rows, heads, hd], cs and sn [rows, 1, rot / 2]."""
    r = x[..., :rot]
    a, b = (r[..., :rot // 2], r[..., rot // 2:]) if layout == "half" else (r[..., 0::2], r[..., 1::2])
    lo, hi = a * cs - b * sn, b * cs + a * sn
    turned = torch.cat([lo, hi], -1) if layout == "half" else torch.stack([lo, hi], -1).flatten(-2)
    return torch.cat([turned, x[..., rot:]], -1)


def _plain_read(s, cu, total, first):
    seq, at = _rows(cu, total)
    pos = at if first is None else at + first[seq].long()
    page, slot = s["pages"][seq, pos // s["case"]["page"]].long(), pos % s["case"]["page"]
    out = []
    for name in ("k", "v"):
        vals = s[name][page, :, slot].float() * s[name + "_scale"][page][..., None]
        out.append(vals.to(torch.bfloat16).flatten(1))
    return out


def _plain_append(s):
    c = s["case"]
    n_q, n_kv, hd, page = c["n_q"], c["n_kv"], c["hd"], c["page"]
    rows = s["qkv"].shape[0]
    x = s["qkv"].view(rows, n_q + 2 * n_kv, hd).float()
    seq, at = _rows(s["cu_new"], rows)
    pos = at + s["ctx"][seq].long()
    t = s["table"][pos]
    qk = _rotate(x[:, :n_q + n_kv], t[:, None, :, 0], t[:, None, :, 1], c["rot"], c["layout"]).to(torch.bfloat16)
    q, k = qk[:, :n_q], qk[:, n_q:]
    ids = s["pages"][seq, pos // page].long()
    held = (s["ctx"].long() % page)[:, None]                                   # tokens a sequence's first page holds
    old_ids = s["pages"].gather(1, (s["ctx"].long() // page).clamp(max=s["pages"].shape[1] - 1)[:, None])[:, 0].long()
    slots = torch.arange(page, device=DEV)[None, :]
    for name, new in (("k", k.float()), ("v", x[:, n_q + n_kv:])):
        codes, scale = s[name], s[name + "_scale"]
        peak = torch.zeros_like(scale).scatter_reduce_(0, ids[:, None].expand(-1, n_kv), new.abs().amax(-1), "amax")
        before = torch.zeros_like(scale)
        before[old_ids] = torch.where(held > 0, scale[old_ids], 0.0)
        grown = torch.maximum(before, peak / 127.0)
        touched = torch.zeros(scale.shape[0], dtype=torch.bool, device=DEV)
        touched[ids] = True
        inverse = torch.where(grown >= 2.0 ** -126, 1.0 / grown, 0.0)
        again = codes[old_ids].float() * (before * inverse)[old_ids][..., None, None]
        again = again.round().clamp(-127, 127).to(torch.int8)
        moved = slots < held                                                   # (a case adds a token at least)
        codes[old_ids] = torch.where(moved[:, None, :, None], again, codes[old_ids])
        codes[ids, :, pos % page] = (new * inverse[ids][..., None]).round().clamp(-127, 127).to(torch.int8)
        scale.copy_(torch.where(touched[:, None], grown, scale))
    kb, vb = _plain_read(s, s["cu_back"], s["n_back"], s["first"])
    return dict(q=q.flatten(1), k=k.flatten(1), cached_k=kb, cached_v=vb, k_scale=s["k_scale"], v_scale=s["v_scale"])


def _plain_gather(s):
    k, v = _plain_read(s, s["cu"], s["total"], None)
    return dict(k=k, v=v)


def _softmax_times(scores, values):
    """scores [..., rows, keys] with -inf where masked (overwritten), values [..., keys, hd]: the weighted mean and the
    logarithm of the sum; a row without keys gives 0 and -inf."""
    top = scores.amax(-1, keepdim=True)
    safe = torch.where(top == -math.inf, 0.0, top)
    p = scores.sub_(safe).exp_()
    total = p.sum(-1, keepdim=True)
    o = torch.matmul(p, values) / torch.where(total == 0, 1.0, total)
    return o, (safe + total.log())[..., 0]


def _plain_decode(s):
    c = s["case"]
    n, n_kv, hd, page = c["n_seqs"], c["n_kv"], c["hd"], c["page"]
    ids = s["pages"].long()
    width = ids.shape[1] * page

    def values(name):
        x = s[name][ids].float() * s[name + "_scale"][ids][..., None, None]     # [seqs, pages, heads, page, hd]
        return x.transpose(1, 2).reshape(n, n_kv, width, hd)

    q = s["q"].float().view(n, n_kv, c["n_q"] // n_kv, hd)
    scores = torch.matmul(q, values("k").transpose(-1, -2)).mul_(hd ** -0.5)
    beyond = torch.arange(width, device=DEV)[None, :] >= s["lens"][:, None]
    o, lse = _softmax_times(scores.masked_fill_(beyond[:, None, None, :], -math.inf), values("v"))
    return dict(o=o.reshape(n, -1).to(torch.bfloat16), lse=lse.reshape(n, -1))


def _plain_prompt(s):
    c = s["case"]
    n, n_q, n_kv, hd = c["n_seqs"], c["n_q"], c["n_kv"], c["hd"]
    tq, tk, mq, mk = s["q"].shape[0], s["k"].shape[0], s["max_q"], s["max_k"]
    at_q = (s["cu_q"][:-1, None].long() + torch.arange(mq, device=DEV)).clamp(max=tq - 1)
    at_k = (s["cu_k"][:-1, None].long() + torch.arange(mk, device=DEV)).clamp(max=tk - 1)
    q = s["q"].float()[at_q].view(n, mq, n_kv, n_q // n_kv, hd).permute(0, 2, 3, 1, 4).reshape(n, n_kv, -1, hd)
    k = s["k"].float()[at_k].view(n, mk, n_kv, hd).transpose(1, 2)
    v = s["v"].float()[at_k].view(n, mk, n_kv, hd).transpose(1, 2)
    scores = torch.matmul(q, k.transpose(-1, -2)).mul_(hd ** -0.5)
    len_q, len_k = s["cu_q"][1:] - s["cu_q"][:-1], s["cu_k"][1:] - s["cu_k"][:-1]
    last = torch.arange(mq, device=DEV)[None, :] + (len_k - len_q)[:, None]                # the last key a query sees
    hidden = torch.arange(mk, device=DEV) > torch.minimum(last, len_k[:, None] - 1)[..., None]
    scores.view(n, n_kv, -1, mq, mk).masked_fill_(hidden[:, None, None], -math.inf)
    o, lse = _softmax_times(scores, v)
    seq, at = _rows(s["cu_q"], tq)
    o = o.view(n, n_q, mq, hd)[seq, :, at].to(torch.bfloat16)
    return dict(o=o.flatten(1), lse=lse.view(n, n_q, mq)[seq, :, at])


_plain = dict(append=_plain_append, gather=_plain_gather, decode=_plain_decode, prompt=_plain_prompt)


# ------------------------------------------------------------------------------------------------ in 64 bits
def exact(case, seed):
    s = prepare(case, seed)
    return dict(append=_exact_append, gather=_exact_gather, decode=_exact_decode, prompt=_exact_prompt)[case["kind"]](case, s)


def _attend(q, k, v, seen):
    """q [heads, rows, hd], k and v [keys, hd], seen [rows, keys]: softmax attention of float64 values."""
    z = torch.einsum("hrd,td->hrt", q, k) / math.sqrt(q.shape[-1])
    z = z.masked_fill(~seen, -math.inf)
    lse = torch.logsumexp(z, -1)
    w = torch.exp(z - torch.where(lse == -math.inf, 0.0, lse)[..., None])
    return torch.einsum("hrt,td->hrd", w, v), lse


def _exact_prompt(case, s):
    n_q, n_kv, hd, L = case["n_q"], case["n_kv"], case["hd"], _lengths(case)
    g = n_q // n_kv
    o = torch.zeros((s["q"].shape[0], n_q, hd), dtype=torch.float64, device=DEV)
    lse = torch.zeros(o.shape[:2], dtype=torch.float64, device=DEV)
    a = b = 0
    for nq, nk in zip(L["q"], L["k"]):
        seen = torch.arange(nk, device=DEV)[None, :] <= torch.arange(nq, device=DEV)[:, None] + (nk - nq)
        for h in range(n_kv):
            q = s["q"][a:a + nq].double().view(nq, n_q, hd)[:, h * g:(h + 1) * g].transpose(0, 1)
            k, v = (s[x][b:b + nk, h * hd:(h + 1) * hd].double() for x in "kv")
            y, z = _attend(q, k, v, seen)
            o[a:a + nq, h * g:(h + 1) * g] = y.transpose(0, 1)
            lse[a:a + nq, h * g:(h + 1) * g] = z.transpose(0, 1)
        a, b = a + nq, b + nk
    return dict(o=o.flatten(1), lse=lse)


def _tokens(s, name, seq, first, count):
    """Tokens first .. first + count of a sequence as float64 values [count, heads, hd]."""
    page = s["case"]["page"]
    pos = torch.arange(first, first + count, device=DEV)
    ids = s["pages"][seq, pos // page].long()
    return s[name][ids, :, pos % page].double() * s[name + "_scale"][ids].double()[..., None]


def _exact_gather(case, s):
    return {x: torch.cat([_tokens(s, x, i, 0, n) for i, n in enumerate(_lengths(case)["len"])]).flatten(1) for x in "kv"}


def _exact_decode(case, s):
    n_q, n_kv, hd = case["n_q"], case["n_kv"], case["hd"]
    g, o, lse = n_q // n_kv, [], []
    for i, n in enumerate(_lengths(case)["len"]):
        k, v, q = _tokens(s, "k", i, 0, n), _tokens(s, "v", i, 0, n), s["q"][i].double().view(n_kv, g, hd)
        seen = torch.ones((1, n), dtype=torch.bool, device=DEV)
        parts = [_attend(q[h][:, None], k[:, h], v[:, h], seen) for h in range(n_kv)]
        o.append(torch.cat([p[0][:, 0] for p in parts]).flatten())
        lse.append(torch.cat([p[1][:, 0] for p in parts]))
    return dict(o=torch.stack(o), lse=torch.stack(lse))


def _exact_append(case, s):
    n_q, n_kv, hd, page, rot, L = case["n_q"], case["n_kv"], case["hd"], case["page"], case["rot"], _lengths(case)
    x = s["qkv"].double().view(-1, n_q + 2 * n_kv, hd)
    turned, a = [], 0
    scales = {n: s[n + "_scale"].double().clone() for n in "kv"}
    back = dict(k=[], v=[])
    for i, (new, ctx) in enumerate(zip(L["new"], L["ctx"])):
        t = s["table"][ctx:ctx + new].double()
        z = torch.complex(t[..., 0], t[..., 1])[:, None]
        y = x[a:a + new, :n_q + n_kv].clone()
        if case["layout"] == "half":
            w = torch.complex(y[..., :rot // 2], y[..., rot // 2:rot]) * z
            y[..., :rot // 2], y[..., rot // 2:rot] = w.real, w.imag
        else:
            y[..., :rot] = torch.view_as_real(torch.view_as_complex(y[..., :rot].reshape(new, -1, rot // 2, 2)) * z).flatten(-2)
        turned.append(y)
        added = dict(k=y[:, n_q:].to(torch.bfloat16).double(), v=x[a:a + new, n_q + n_kv:])
        for p in range(ctx // page, -(-(ctx + new) // page)):
            lo, hi = max(ctx, p * page), min(ctx + new, (p + 1) * page)
            at = int(s["pages"][i, p])
            for n in "kv":
                v = added[n][lo - ctx:hi - ctx]
                held = s[n][at, :, :lo - p * page].double().transpose(0, 1)
                before = scales[n][at] if lo > p * page else torch.zeros(n_kv, dtype=torch.float64, device=DEV)
                scale = torch.maximum(before, v.abs().amax((0, 2)) / 127)
                inv = torch.where(scale > 0, 1 / scale, 0.0)[None, :, None]
                codes = torch.cat([held * (before[None, :, None] * inv), v * inv]).round().clamp(-127, 127)
                back[n].append(codes * scale[None, :, None])
                scales[n][at] = scale
        a += new
    y = torch.cat(turned)
    return dict(q=y[:, :n_q].flatten(1), k=y[:, n_q:].flatten(1), cached_k=torch.cat(back["k"]).flatten(1),
                cached_v=torch.cat(back["v"]).flatten(1), k_scale=scales["k"], v_scale=scales["v"])
