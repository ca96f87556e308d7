"""Helpers for the tests of the paged cache in 4 bits: caches as the oracle has them, the same on the GPU, and how far attention over them may be from 64 bits."""
from __future__ import annotations

import numpy as np

import paper_2503_01873_amd as P
from oracle import cache4_oracle as c4
from tests import cache_bounds as cb
from tests import cache_harness as ch


def empty(g, S, Hkv, d, page, width, spare=2, shift=False, mean=True):
    """A cache that holds nothing: every byte and scale is what must not be looked at."""
    pages = S * width + spare
    raw = page * d * 17 // 32
    return {"k": np.full((pages, Hkv, raw), 0xFF, np.uint8), "v": np.full((pages, Hkv, raw), 0x7F, np.uint8),
            "kscale": np.full((pages, Hkv, page), np.nan, np.float32), "vscale": np.full((pages, Hkv, page), np.nan, np.float32),
            "kmean": np.full((pages, Hkv, d), np.nan, np.float32) if mean else None,
            "kshift": (3 * g.standard_normal((Hkv, d))).astype(np.float32) if shift else None,
            "table": g.permutation(pages)[:S * width].reshape(S, width).astype(np.int32), "length": np.zeros(S, np.int32), "format": "i4"}


def filled(g, lengths, Hkv, d, page, dtype="f16", width=None, wild=False, **kw):
    """A cache whose sequences hold `lengths` tokens.  wild: magnitudes that differ by 2^10 from token to token and by 2^6 from group to group of channels."""
    S = len(lengths)
    width = width or max(1, -(-max(lengths) // page))
    c = empty(g, S, Hkv, d, page, width, **kw)
    c["length"] = np.array(lengths, np.int32)
    R = int(sum(lengths))
    k, v = g.standard_normal((R, Hkv, d)), g.standard_normal((R, Hkv, d))
    if wild:
        v *= 2.0 ** g.integers(-5, 6, (R, Hkv, 1)) * np.repeat(2.0 ** g.integers(-6, 1, (R, Hkv, d // 32)), 32, 2)
        k *= 2.0 ** g.integers(-2, 3, (R, Hkv, 1)) * np.repeat(2.0 ** g.integers(-3, 1, (R, Hkv, d // 32)), 32, 2)
    if c["kshift"] is not None:
        k += c["kshift"]
    if R:
        c4.write(c, ch.rounded(k, dtype), ch.rounded(v, dtype), ch.starts(lengths))
    return c


class OnGpu:
    """The buffers of a cache on the GPU, and its description."""

    def __init__(self, c, device="cuda:0"):
        import torch
        self.t = {n: torch.from_numpy(np.ascontiguousarray(x)).to(device) for n, x in c.items() if isinstance(x, np.ndarray)}
        page, d = c4.sizes(c)
        self.cache = P.pasa_cache(*(self.t[n] for n in ("k", "v", "kscale", "vscale", "table", "length")), S=len(c["length"]), Hkv=c["k"].shape[1], d=d,
                                  page=page, pages=c["k"].shape[0], table_width=c["table"].shape[1], format=P.CACHE_I4,
                                  kmean=self.t.get("kmean"), kshift=self.t.get("kshift"))

    def back(self, name):
        return self.t[name].cpu().numpy()


def attend(c, q, row_start, scale, dtype, tree=None, blocks=None):
    """(o, bound) of every row and head, float64; rows of no sequence are NaN.

    An output is sum P v / sum P.  Keys and values come as factor * code times the scale: whole numbers below 2^11, which fp16 holds, so nothing of them is rounded.
    Of each P: its exponent carries the score (sums of d products in fp32 in any order, d 2^-24 of the sum of their magnitudes), a rounding each of the factor
    ks * scale, of the sum with log2 of the value's scale and of the difference from the level (3 2^-24 of numbers below 2 size log2(e) + 128: logarithms of
    scales lie within 128), and 2^-21 for the logarithm and the exponential; numerator and denominator carry it.  In the numerator P is an fp16
    number: half a step, 2^-11 of it, or, below 2^-14, 2^-25; the row's largest P is 2^7 at least in any wavefront's level, so the latter is 2^-32 of the
    largest product of P and scale that the row sees, times a number (1568 at most), for each token.  Both sums are of fp32: a lane adds at most a fourth of the
    tokens in turn, and what wavefronts and workgroups hold (at most 64 additions more).  The type of the output rounds once."""
    p_c = c4.plain(c)
    R, Hq, d = q.shape
    G = Hq // c["k"].shape[1]
    o, bound = np.full((R, Hq, d), np.nan), np.full((R, Hq, d), np.nan)
    for r, h, k, v, s in cb._seen(p_c, row_start, R, tree, blocks):
        for i in range(h * G, (h + 1) * G):
            with np.errstate(all="ignore"):
                x = (k @ q[r, i]) * scale
                if not len(x) or x.max() == -np.inf:
                    o[r, i], bound[r, i] = 0.0, 0.0
                    continue
                p = np.exp(x - x.max())
                p /= p.sum()
                size = (np.abs(k) @ np.abs(q[r, i])).max() * scale
                e = (d + 6) * 2.0 ** -24 * size + 128 * 3 * 2.0 ** -24 + 2.0 ** -21
                sums = (len(x) / 4 + 64) * 2.0 ** -24
                o[r, i], wide = p @ v, p @ np.abs(v)
                bound[r, i] = (2.0 ** -11 + 2 * e + sums) * wide + (2 * e + sums + ch.HALF_STEP[dtype]) * np.abs(o[r, i]) + \
                    len(x) * 2.0 ** -32 * (p * s).max() * 1568 + cb.SMALLEST[dtype]
    return o, bound


def check(got, ref):
    o, bound = ref
    assert np.array_equal(np.isnan(got), np.isnan(o)), "other rows are NaN"
    with np.errstate(invalid="ignore"):
        off = np.abs(got - o) / np.maximum(bound, 1e-300)
    assert not (off > 1.0).any(), (float(np.nanmax(off)), np.unravel_index(np.nanargmax(off), off.shape))
