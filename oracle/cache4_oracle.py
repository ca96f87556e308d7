"""CPU oracle of the paged cache in 4 bits, from the definition of PASA_CACHE_I4 in include/pasa.h, in fp64 numpy.  Test infrastructure only.

A cache here is a dict as in cache_oracle, with k, v uint8 [pages, Hkv, page * d * 17 / 32] as the library holds them and format "i4".  `plain` gives the
same cache with k, v as the whole numbers factor * code [pages, Hkv, page, d], which cache_oracle's read, choose and attend take.
"""
from __future__ import annotations

from fractions import Fraction

import numpy as np

from . import cache_oracle as co

GROUP = 32


def _nearest(x, unit):
    """The whole number nearest to x / unit, ties to even.  x, unit >= 0 in fp64: unit has 16 bits, so (n + 1/2) unit is exact."""
    n = np.floor(x / unit)
    n = np.where(n * unit > x, n - 1, n)
    n = np.where((n + 1) * unit <= x, n + 1, n)
    middle = (n + 0.5) * unit
    return np.where((x > middle) | ((x == middle) & (n % 2 == 1)), n + 1, n)


def scale_of(top):
    """The least number of 8 significant bits that is not below top / 1568, by fractions."""
    want = Fraction(float(top)) / 1568
    e = 0
    while Fraction(2) ** (e + 1) <= want:
        e += 1
    while Fraction(2) ** e > want:
        e -= 1
    step = Fraction(2) ** (e - 7)
    return float(-(-want // step) * step)


def encode(x):
    """x float32 [..., d] -> codes int8 -7 .. 7, factors uint8 [..., d / 32], scales float32."""
    x = np.asarray(x, np.float32).astype(np.float64)
    bad = ~np.isfinite(x).all(-1)
    x = np.where(bad[..., None], 0.0, x)
    top = np.abs(x).max(-1)
    small = top < 2.0 ** -98
    unique, at = np.unique(np.where(small, 1.0, top), return_inverse=True)
    scale = np.array([scale_of(t) for t in unique])[at].reshape(top.shape)
    scale = np.where(small, 1.0, scale)
    parts = x.reshape(*x.shape[:-1], -1, GROUP)
    factor = np.maximum(_nearest(np.abs(parts).max(-1), 7 * scale[..., None]), 1)
    assert factor.size == 0 or factor.max() <= 224
    code = np.minimum(_nearest(np.abs(parts), (factor * scale[..., None])[..., None]), 7) * np.sign(parts)
    return code.reshape(x.shape).astype(np.int8), factor.astype(np.uint8), np.where(bad, np.nan, scale).astype(np.float32)


def sizes(c):
    """page, d"""
    page = c["kscale"].shape[2]
    return page, c["k"].shape[2] * 32 // (17 * page)


def numbers(c, which):
    """factor * code of all pages, int64 [pages, Hkv, page, d]"""
    page, d = sizes(c)
    raw = c[which].astype(np.int64)
    codes, factor = raw[..., :page * d // 2], raw[..., page * d // 2:]
    code = np.stack([codes & 15, codes >> 4], -1).reshape(*raw.shape[:2], page, d) - 8
    return code * np.repeat(factor.reshape(*raw.shape[:2], page, d // GROUP), GROUP, -1)


def plain(c):
    return {**c, "k": numbers(c, "k"), "v": numbers(c, "v")}


def put(c, which, i, h, t, code, factor):
    """A token's codes and factors into page i."""
    page, d = sizes(c)
    code = code.astype(np.int64) + 8
    c[which][i, h, t * d // 2:(t + 1) * d // 2] = code[0::2] | code[1::2] << 4
    c[which][i, h, page * d // 2 + t * d // GROUP:page * d // 2 + (t + 1) * d // GROUP] = factor


def write(c, k, v, row_start):
    """Tokens enter; c is changed.  k, v float32 [R, Hkv, d]."""
    page, d = sizes(c)
    shift = 0 if c["kshift"] is None else c["kshift"]
    new = {"k": encode(np.float32(k) - np.float32(shift)), "v": encode(v)}
    touched = set()
    table_of = {"k": c["kscale"], "table": c["table"]}                   # what co._page looks at
    for b, n, r0, m in co._spans({**c, "k": np.empty((0, 0, page, 0))}, row_start, len(k)):
        for t in range(m):
            pos = n - m + t
            i = co._page(table_of, b, pos // page) if pos >= 0 else None
            if i is None:
                continue
            touched.add((i, min(page, n - pos // page * page)))
            for which, (code, factor, scale) in new.items():
                for h in range(k.shape[1]):
                    put(c, which, i, h, pos % page, code[r0 + t, h], factor[r0 + t, h])
                c[which + "scale"][i, :, pos % page] = scale[r0 + t]
    if c["kmean"] is not None:
        x = numbers(c, "k")
        for i, left in touched:
            c["kmean"][i] = co.values(x[i, :, :left], c["kscale"][i, :, :left], "i4").mean(1).astype(np.float32)
