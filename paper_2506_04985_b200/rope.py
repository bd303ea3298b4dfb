"""Tables of rotary positions for fpt_rope_append (offline helper, numpy float64).

A pair i of a head (i < rot_dim / 2) turns by the angle p f_i at position p.  The angles are formed and their cosines and sines taken
in float64, so that far positions keep their 24 bits; the table is float32.  What a long-context model changes is f_i (and, with the
last of the schemes, a factor on cosine and sine); the scheme is an argument here, the kernel reads a table:

    none       f_i = base^(-2 i / rot_dim)
    linear     f_i / factor                                            (position interpolation)
    ntk        base replaced by base factor^(rot_dim / (rot_dim - 2))    (the lowest frequency is divided by factor)
    by_parts   f_i kept where its wave length 2 pi / f_i is below original / high, divided by factor where it is above
               original / low, and in between  ((1 - s) / factor + s) f_i,  s = (original / wave - low) / (high - low)
    yarn       the same between the pairs that turn beta_fast and beta_slow times within `original` positions, on a ramp over the pair's number;
               cosine and sine times 0.1 ln(factor) + 1
"""
import math

import numpy as np


def frequencies(rot_dim, base=10000.0, scheme="none", factor=1.0, original=8192, low=1.0, high=4.0, beta_fast=32.0, beta_slow=1.0):
    """(f float64 [rot_dim / 2], factor on cosine and sine)."""
    if rot_dim <= 0 or rot_dim % 2 or base <= 0 or factor < 1:
        raise ValueError("rope: an even positive rot_dim, a positive base and a factor of at least 1 are wanted")
    i = np.arange(rot_dim // 2, dtype=np.float64)
    if scheme == "ntk":
        if rot_dim < 4:
            raise ValueError("rope: ntk needs two pairs")
        base = base * factor ** (rot_dim / (rot_dim - 2))
    f = base ** (-2.0 * i / rot_dim)
    if scheme in ("none", "ntk"):
        return f, 1.0
    if scheme == "linear":
        return f / factor, 1.0
    if scheme == "by_parts":
        s = np.clip((original * f / (2 * math.pi) - low) / (high - low), 0.0, 1.0)
        return ((1 - s) / factor + s) * f, 1.0
    if scheme == "yarn":
        def pair_of(turns):                                 # the pair that turns so often within `original` positions
            return rot_dim * math.log(original / (2 * math.pi * turns)) / (2 * math.log(base))
        first, last = max(math.floor(pair_of(beta_fast)), 0), min(math.ceil(pair_of(beta_slow)), rot_dim - 1)
        s = 1 - np.clip((i - first) / max(last - first, 1e-3), 0.0, 1.0)
        return ((1 - s) / factor + s) * f, 0.1 * math.log(factor) + 1.0 if factor > 1 else 1.0
    raise ValueError(f"rope: unknown scheme {scheme!r}")


def rope_table(n_pos, rot_dim, base=10000.0, scheme="none", first=0, **scaling):
    """float32 [n_pos, rot_dim / 2, 2]: cosine and sine of positions first .. first + n_pos - 1."""
    f, gain = frequencies(rot_dim, base, scheme, **scaling)
    angle = np.arange(first, first + n_pos, dtype=np.float64)[:, None] * f
    return np.stack([np.cos(angle) * gain, np.sin(angle) * gain], -1).astype(np.float32)
