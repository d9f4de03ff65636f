"""fp64 definition of the 4-bit node states.

TEST INFRASTRUCTURE ONLY (see the package docstring).

64 neighbouring entries of one token and KV head form a group.  lo is its least entry, s the bf16 number
nearest to (hi - lo) / 16 (ties to even), an entry's code floor((x - lo) / s) held within 0..15 (0 where s
is 0), and what it stands for lo + s (code + 1/2) (lo where s is 0).  The quotient is the exact one: what fp64 rounds
off a difference or a quotient next to a border of two cells is put right.
"""
from __future__ import annotations

import numpy as np

GROUP = 64


def round_to_bf16(x):
    """The bf16 number nearest to x (ties to even; finite), as fp64: 8 significant bits, and no finer than the
    subnormals' step 2^-133."""
    x = np.asarray(x, np.float64)
    _, e = np.frexp(x)
    e = np.maximum(e - 8, -133)
    return np.ldexp(np.rint(np.ldexp(x, -e)), e)


def encode(x):
    """x fp64 [..., D] (bf16 numbers): (codes int [..., D], s [..., D / 64], lo [..., D / 64])."""
    g = x.reshape(x.shape[:-1] + (x.shape[-1] // GROUP, GROUP))
    lo, hi = g.min(-1), g.max(-1)
    s = round_to_bf16((hi - lo) / 16)
    lo1, s1 = lo[..., None], s[..., None]
    d = g - lo1
    b = g - d
    lost = (g - (d + b)) + (b - lo1)               # g - lo = d + lost
    with np.errstate(divide="ignore", invalid="ignore"):
        c = np.clip(np.floor(d / s1), 0, 16)
        rest = d - c * s1                          # exact: c s is a few whole steps of s
        c = c - ((rest < 0) | ((rest == 0) & (lost < 0)))
    c = np.where(s[..., None] > 0, np.clip(c, 0, 15), 0).astype(np.int64)
    return c.reshape(x.shape), s, lo


def values(x):
    """What the 4-bit form of x stands for, fp64."""
    c, s, lo = encode(x)
    c = c.reshape(x.shape[:-1] + (x.shape[-1] // GROUP, GROUP))
    v = np.where(s[..., None] > 0, lo[..., None] + s[..., None] * (c + 0.5), lo[..., None])
    return v.reshape(x.shape)
