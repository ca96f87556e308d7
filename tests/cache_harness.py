"""Helpers for the tests of the paged cache: caches in numpy as the oracle has them, and the same on the GPU."""
from __future__ import annotations

import numpy as np

import paper_2503_01873_amd as P
from oracle import cache_oracle as co

FORMAT = {"i8": P.CACHE_I8, "e4m3": P.CACHE_E4M3}
IO = {"f16": P.IO_F16, "bf16": P.IO_BF16}
HALF_STEP = {"f16": 2.0 ** -11, "bf16": 2.0 ** -8}       # of a value that is rounded to the type, relative
TINY = {"f16": 2.0 ** -25, "bf16": 0.0}                  # half a step of the smallest fp16 values


def rounded(x, dtype):
    """x as values of the type, in float32."""
    if dtype == "f16":
        return np.asarray(x, np.float32).astype(np.float16).astype(np.float32)
    u = np.asarray(x, np.float32).view(np.uint32)
    return ((u + 0x7FFF + ((u >> 16) & 1)) & np.uint32(0xFFFF0000)).view(np.float32)


def starts(rows):
    return np.concatenate([[0], np.cumsum(rows)]).astype(np.int32)


def empty(g, S, Hkv, d, page, width, format, spare=2, shift=False, mean=True):
    """A cache that holds nothing: every byte and scale is what must not be looked at."""
    pages = S * width + spare
    c = {"k": np.full((pages, Hkv, page, d), 0x7F, np.uint8), "v": np.full((pages, Hkv, page, d), 0xFF, np.uint8),
         "kscale": np.full((pages, Hkv, page), np.nan, np.float32), "vscale": np.full((pages, Hkv, page), np.nan, np.float32),
         "kmean": np.full((pages, Hkv, d), np.nan, np.float32) if mean else None,
         "kshift": (3 * g.standard_normal((Hkv, d))).astype(np.float32) if shift else None,
         "table": g.permutation(pages)[:S * width].reshape(S, width).astype(np.int32),
         "length": np.zeros(S, np.int32), "format": format}
    return c


def filled(g, lengths, Hkv, d, page, format, dtype="f16", width=None, wild=False, **kw):
    """A cache whose sequences hold `lengths` tokens.  wild: magnitudes of keys and values that differ by 2^10 from token to token."""
    S = len(lengths)
    width = width or max(1, -(-max(lengths) // page))
    c = empty(g, S, Hkv, d, page, width, format, **kw)
    c["length"] = np.array(lengths, np.int32)
    R = int(sum(lengths))
    k, v = g.standard_normal((R, Hkv, d)), g.standard_normal((R, Hkv, d))
    if wild:
        v *= 2.0 ** g.integers(-5, 6, (R, Hkv, 1))
        k *= 2.0 ** g.integers(-2, 3, (R, Hkv, 1))
    if c["kshift"] is not None:
        k += c["kshift"]
    if R:
        co.write(c, rounded(k, dtype), rounded(v, dtype), starts(lengths))
    return c


class OnGpu:
    """The buffers of a cache on the GPU, and its description."""

    def __init__(self, c, device="cuda:0"):
        import torch
        self.t = {n: torch.from_numpy(np.ascontiguousarray(x)).to(device) for n, x in c.items() if isinstance(x, np.ndarray)}
        pages, Hkv, page, d = c["k"].shape
        self.cache = P.pasa_cache(*(self.t[n] for n in ("k", "v", "kscale", "vscale", "table", "length")), S=len(c["length"]), Hkv=Hkv, d=d,
                                  page=page, pages=pages, table_width=c["table"].shape[1], format=FORMAT[c["format"]],
                                  kmean=self.t.get("kmean"), kshift=self.t.get("kshift"))

    def back(self, name):
        return self.t[name].cpu().numpy()


def tensor(x, dtype, stride=None, device="cuda:0"):
    """Rows of a type on the GPU, `stride` elements apart (what is between them is NaN)."""
    import torch
    t = torch.from_numpy(np.ascontiguousarray(x, np.float32)).to(device).to(torch.float16 if dtype == "f16" else torch.bfloat16)
    n = t[0].numel() if len(t) else int(np.prod(x.shape[1:]))
    if stride is None or stride == n:
        return t, n
    wide = torch.full((len(t), stride), float("nan"), dtype=t.dtype, device=device)
    wide[:, :n] = t.view(len(t), n)
    return wide, stride


def ints(x, device="cuda:0"):
    import torch
    return torch.from_numpy(np.asarray(x, np.int32)).to(device)


def run_attend(gpu, q, row_start, scale, dtype, tree=None, blocks=None, stride=None, stream=None, o=None):
    """o as float64 [R, Hq, d], rows that were not written NaN; nothing behind them is written."""
    import torch
    R, Hq, d = q.shape
    dev = gpu.t["k"].device
    tq, stride = tensor(q, dtype, stride, dev)
    flat = torch.full((R * Hq * d + 4096,), float("nan"), dtype=tq.dtype, device=dev)
    need = P.pasa_attn_cache_workspace(gpu.cache, R, Hq)
    assert need > 0
    ws = torch.full((need + 4096,), 0xFF, dtype=torch.uint8, device=dev)         # NaN everywhere
    tt = None if tree is None else torch.from_numpy(np.asarray(tree, np.uint64).view(np.int64)).to(dev)
    tb = None if blocks is None else ints(blocks, dev)
    P.pasa_attn_cache(gpu.cache, tq, flat, R, stride, ints(row_start, dev), Hq, scale, ws, need, stream or torch.cuda.current_stream(dev), tree=tt,
                      blocks=tb, count=0 if blocks is None else blocks.shape[2], io_dtype=IO[dtype])
    torch.cuda.synchronize(dev)
    assert bool(torch.isnan(flat[R * Hq * d:]).all()) and bool((ws[need:] == 0xFF).all()), "written behind the end"
    return flat[:R * Hq * d].view(R, Hq, d).double().cpu().numpy()


def attend_bound(c, ref, dtype, keys):
    """How far an output may be from the oracle's, by element.

    P: one rounding to fp16, half a step is 2^-11 of it; its exponent carries the score (sums of d products in fp32 in any order: d 2^-24 of the sum of
    magnitudes), one rounding each of the factor, the sum with log2 of the value's scale and the difference from the level (3 2^-24 of numbers
    below 2 size log2(e) + 64), that logarithm and the exponential itself (2^-21 allows the hardware's 1 ulp of each).  Numerator and
    denominator each carry it.  P below 2^-14 keeps 2^-25 of the level: at most 2^-25 times a code's magnitude times the largest
    scale for every key.  The type of the output rounds once."""
    o, wide, size = ref
    d = c["k"].shape[3]
    e = ((d + 6) * 2.0 ** -24 * size + 64 * 3 * 2.0 ** -24 + 2.0 ** -21)[..., None]
    with np.errstate(invalid="ignore"):
        most = np.nanmax(np.where(np.isfinite(c["vscale"]), c["vscale"], 0)) * (127 if c["format"] == "i8" else 448)
        lost = keys * 2.0 ** -25 * most
        return (2.0 ** -11 + 2 * e) * wide + 2 * e * np.abs(o) + lost + HALF_STEP[dtype] * np.abs(o) + TINY[dtype] + 1e-30


def check_attend(c, got, ref, dtype, keys):
    o = ref[0]
    assert np.array_equal(np.isnan(got), np.isnan(o)), "other rows are NaN"
    bound = attend_bound(c, ref, dtype, keys)
    with np.errstate(invalid="ignore"):
        off = np.abs(got - o)
        worst = np.nanmax(off / bound) if np.isfinite(o).any() else 0.0
    assert worst <= 1.0, (worst, float(np.nanmax(off)))
