"""How far attention over the paged cache may be from 64 bits, row by row: by the products that a row itself sees, and by how many they are."""
from __future__ import annotations

import numpy as np

from oracle import cache_oracle as co
from tests import cache_harness as ch

SMALLEST = {"f16": 2.0 ** -25, "bf16": 2.0 ** -134}          # half a step of the smallest values of the type


def _seen(c, row_start, R, tree, blocks):
    """(row, KV head, pages' tokens in order as (k, v, scale of v), which of them the row sees), for every row that belongs to a sequence."""
    P, Hkv, page, d = c["k"].shape
    for b, n, r0, m in co._spans(c, row_start, R):
        for h in range(Hkv):
            pos, k, v, s = [np.zeros(0, int)], [np.zeros((0, d))], [np.zeros((0, d))], [np.zeros(0)]
            for p in range(-(-n // page)) if blocks is None else blocks[b, h]:
                i = co._page(c, b, p) if 0 <= p < c["table"].shape[1] else None
                left = min(page, n - int(p) * page)
                if i is None or left <= 0:
                    continue
                pos.append(np.arange(p * page, p * page + left))
                k.append(co.values(c["k"][i, h, :left], c["kscale"][i, h, :left], c["format"]))
                v.append(co.values(c["v"][i, h, :left], c["vscale"][i, h, :left], c["format"]))
                s.append(np.where((v[-1] == 0).all(1) & (c["vscale"][i, h, :left] == 1), 2.0 ** -60, c["vscale"][i, h, :left].astype(np.float64)))
            pos, k, v, s = (np.concatenate(x) for x in (pos, k, v, s))
            for t in range(m):
                nth = pos - (n - m)
                if tree is None:
                    see = nth <= t
                else:
                    bits = np.array([int(tree[r0 + t]) >> j & 1 for j in range(64)], bool)
                    see = (nth < 0) | ((nth < 64) & bits[np.clip(nth, 0, 63)])
                yield r0 + t, h, k[see], v[see], s[see]


def attend(c, q, row_start, scale, dtype, tree=None, blocks=None):
    """(o, bound) of every row and head, float64; rows of no sequence are NaN.

    An output is sum P v / sum P.  Of each P: its exponent carries the score (sums of d products in fp32 in any order, d 2^-24 of the sum of their
    magnitudes), a rounding each of the factor, of the sum with log2 of the value's scale and of the difference from the level (3 2^-24 of numbers below
    2 size log2(e) + 128: logarithms of scales lie within 128), and 2^-21 for the logarithm and the exponential; numerator and denominator carry it.  In the
    numerator P is an fp16 number: half a step, 2^-11 of it, or, below 2^-14, 2^-25; the row's largest P is 2^7 at least in any wavefront's level, so the
    latter is 2^-32 of the largest product of P and scale that the row sees, times a code, for each token.  Both sums are of fp32: a lane adds at most a
    fourth of the tokens in turn, and what wavefronts and workgroups hold (at most 64 additions more).  Products with 2^-14 / scale lose 2^-15 where
    scales exceed 2^110.  The type of the output rounds once."""
    R, Hq, d = q.shape
    G = Hq // c["k"].shape[1]
    o, bound = np.full((R, Hq, d), np.nan), np.full((R, Hq, d), np.nan)
    code = 127 if c["format"] == "i8" else 448
    for r, h, k, v, s in _seen(c, row_start, R, tree, blocks):
        for g in range(h * G, (h + 1) * G):
            x = (k @ q[r, g]) * scale
            if not len(x) or x.max() == -np.inf:
                o[r, g], bound[r, g] = 0.0, 0.0
                continue
            p = np.exp(x - x.max())
            p /= p.sum()
            size = (np.abs(k) @ np.abs(q[r, g])).max() * scale
            e = (d + 6) * 2.0 ** -24 * size + 128 * 3 * 2.0 ** -24 + 2.0 ** -21
            sums = (len(x) / 4 + 64) * 2.0 ** -24 + (2.0 ** -15 if s.max() > 2.0 ** 110 else 0.0)
            o[r, g], wide = p @ v, p @ np.abs(v)
            bound[r, g] = (2.0 ** -11 + 2 * e + sums) * wide + (2 * e + sums + ch.HALF_STEP[dtype]) * np.abs(o[r, g]) + \
                len(x) * 2.0 ** -32 * (p * s).max() * code + SMALLEST[dtype]
    return o, bound


def check(got, ref):
    o, bound = ref
    assert np.array_equal(np.isnan(got), np.isnan(o)), "other rows are NaN"
    with np.errstate(invalid="ignore"):
        off = np.abs(got - o) / np.maximum(bound, 1e-300)
    assert not (off > 1.0).any(), (float(np.nanmax(off)), np.unravel_index(np.nanargmax(off), off.shape))
    # nothing else could pass for it: nearly all bounds lie far below what they are bounds of
    there = np.isfinite(o) & (o != 0)
    assert (bound[there] < 0.25 * np.abs(o[there])).mean() > 0.9
