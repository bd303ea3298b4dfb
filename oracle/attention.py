"""Oracle of the attention between the two attention projections: rotary positions, the append to a paged 8-bit cache,
reading it back, softmax attention.  Written from the formulas of include/fpt.h; numpy, float64 where the formulas fix no
precision, float32 with one rounding per operation where they do."""
import numpy as np

from .bf16 import round_to_bf16

F32 = np.float32


def rope(x, cos_sin, rot, interleaved):
    """x [tokens, heads, hd] float32 (bf16 values), cos_sin [tokens, rot / 2, 2] -> rotated, rounded to bf16 (as float32)."""
    x = x.astype(F32)
    c, s = cos_sin[:, None, :, 0].astype(F32), cos_sin[:, None, :, 1].astype(F32)
    a, b = ((x[..., 0:rot:2], x[..., 1:rot:2]) if interleaved else (x[..., :rot // 2], x[..., rot // 2:rot]))
    lo, hi = a * c - b * s, b * c + a * s
    y = x.copy()
    if interleaved:
        y[..., 0:rot:2], y[..., 1:rot:2] = lo, hi
    else:
        y[..., :rot // 2], y[..., rot // 2:rot] = lo, hi
    return round_to_bf16(y)


def _codes(v):
    with np.errstate(invalid="ignore"):
        return np.where(np.isnan(v), -127, np.clip(np.rint(v), -127, 127)).astype(np.int8)


def append(new, codes, scale, pages, ctx, page):
    """Values new [tokens, heads, hd] (float32) of one sequence behind its ctx tokens; codes [n_pages, heads, page, hd] and scale
    [n_pages, heads] are changed in place."""
    n = new.shape[0]
    for p in range(ctx // page, -(-(ctx + n) // page)):
        lo, hi = max(ctx, p * page), min(ctx + n, (p + 1) * page)
        held, at = lo - p * page, pages[p]
        v = new[lo - ctx:hi - ctx].astype(F32)                             # [tokens, heads, hd]
        with np.errstate(invalid="ignore"):
            m = np.where(np.isfinite(v), np.abs(v), F32(0)).max((0, 2))
        before = scale[at].copy() if held else np.zeros(v.shape[1], F32)
        s = np.maximum(before, (m / F32(127)).astype(F32))
        with np.errstate(divide="ignore", over="ignore", invalid="ignore"):
            inv = np.where(s >= F32(2.0 ** -126), F32(1) / s, F32(0)).astype(F32)
            grown = s > before
            again = _codes(codes[at, :, :held].astype(F32) * (before * inv)[:, None, None])
            codes[at, :, :held] = np.where(grown[:, None, None], again, codes[at, :, :held])
            codes[at, :, held:held + hi - lo] = _codes(v * inv[None, :, None]).transpose(1, 0, 2)
        scale[at] = s


def read(codes, scale, pages, first, count, page):
    """Tokens first .. first + count of one sequence: float32 code * scale [count, heads, hd]."""
    pos = np.arange(first, first + count)
    at = np.asarray(pages)[pos // page]
    return codes[at, :, pos % page].astype(F32) * scale[at][..., None]


def attend(q, k, v, scale, causal):
    """q [len_q, n_q, hd], k and v [len_k, n_kv, hd] (any float): float64 softmax attention of one sequence, the last query seeing
    the last key.  -> (o [len_q, n_q, hd], lse [len_q, n_q], weighted mean of |v| like o, largest sum_d |q_d k_d| * scale like lse)."""
    q, k, v = (np.asarray(t, np.float64) for t in (q, k, v))
    (lq, nq, hd), (lk, nkv) = q.shape, k.shape[:2]
    g = nq // nkv
    o, spread = np.zeros((2, lq, nq, hd))
    lse, mass = np.full((lq, nq), -np.inf), np.zeros((lq, nq))
    seen = np.clip(np.arange(lq) + lk - lq + 1, 0, lk) if causal else np.full(lq, lk)
    mask = np.arange(lk)[None, :] < seen[:, None]
    for h in range(nkv if lq and lk else 0):
        sl = slice(h * g, (h + 1) * g)
        for rows in ([slice(0, lq)] if np.isfinite(k[:, h]).all() and np.isfinite(v[:, h]).all() else
                     [slice(i, i + 1) for i in range(lq)]):             # one at a time: what is hidden is left out, not weighted
            n = int(seen[rows].max())
            if n == 0:
                continue
            qs, ks, vs = q[rows, sl].transpose(1, 0, 2), k[:n, h], v[:n, h]
            with np.errstate(invalid="ignore", over="ignore", divide="ignore"):
                z = np.where(mask[rows, :n], qs @ ks.T * scale, -np.inf)
                top = np.maximum(z.max(-1, keepdims=True), -1e300)
                w = np.exp(z - top)
                total = w.sum(-1, keepdims=True)
                p = w / np.where(total == 0, 1, total)
                o[rows, sl] = (p @ vs).transpose(1, 0, 2)
                spread[rows, sl] = (p @ np.abs(vs)).transpose(1, 0, 2)
                lse[rows, sl] = np.where(total == 0, -np.inf, top + np.log(total))[..., 0].T
                mass[rows, sl] = np.where(mask[rows, :n], np.abs(qs) @ np.abs(ks).T, 0).max(-1).T * scale
    return o, lse, spread, mass
