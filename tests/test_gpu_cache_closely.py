"""Attention over the paged cache against 64 bits, each row within what its own products allow."""
import numpy as np
import pytest

from oracle import cache_oracle as co
from tests import cache_bounds as cb
from tests import cache_harness as ch

pytestmark = pytest.mark.gpu


def _check(c, q, rows, dtype="f16", scale=None, **kw):
    scale = float(np.float32(q.shape[2] ** -0.5 if scale is None else scale))
    got = ch.run_attend(ch.OnGpu(c), q, ch.starts(rows), scale, dtype, **kw)
    cb.check(got, cb.attend(c, q, ch.starts(rows), scale, dtype, **kw))


def _queries(g, R, Hq, d, dtype, size):
    return ch.rounded(size * g.standard_normal((R, Hq, d)), dtype).astype(np.float64)


@pytest.mark.parametrize("format,dtype", [("i8", "f16"), ("e4m3", "bf16"), ("i8", "bf16"), ("e4m3", "f16")])
@pytest.mark.parametrize("Hq,Hkv,d", [(28, 4, 128), (5, 5, 64), (16, 2, 64)])
@pytest.mark.parametrize("size", [0.5, 4.0])
def test_steps(Hq, Hkv, d, format, dtype, size):
    """Weights spread over all keys, or on a few; lengths around the units of work."""
    g = np.random.default_rng([41, Hq, d])
    lengths = [1, 2, 63, 64, 65, 700, 128, 1345, 0, 5000]
    c = ch.filled(g, lengths, Hkv, d, 64, format, dtype, wild=True)
    _check(c, _queries(g, len(lengths), Hq, d, dtype, size), [1] * len(lengths), dtype)


@pytest.mark.parametrize("format", ["i8", "e4m3"])
@pytest.mark.parametrize("Hq,Hkv,d", [(28, 4, 128), (4, 4, 64)])
@pytest.mark.parametrize("tree", [False, True])
def test_chains_and_trees(Hq, Hkv, d, tree, format):
    g = np.random.default_rng([42, Hq, d])
    lengths, rows = [300, 64, 5, 90, 1, 2000], [7, 64, 9, 0, 1, 40]
    c = ch.filled(g, lengths, Hkv, d, 32, format, wild=True)
    bits = None
    if tree:
        bits = g.integers(0, 1 << 63, sum(rows)).astype(np.uint64) | np.concatenate([np.uint64(1) << np.arange(n, dtype=np.uint64) for n in rows])
    _check(c, _queries(g, sum(rows), Hq, d, "f16", 1.5), rows, tree=bits)


@pytest.mark.parametrize("page,count", [(16, 9), (64, 4), (128, 2)])
def test_chosen_pages(page, count):
    g = np.random.default_rng([43, page])
    lengths, Hq, Hkv, d = [900, 33, 640, 1000], 12, 2, 128
    c = ch.filled(g, lengths, Hkv, d, page, "i8", wild=True)
    blocks = np.full((4, Hkv, count), -1, np.int32)
    for b, n in enumerate(lengths):
        for h in range(Hkv):
            at = np.sort(g.permutation(-(-n // page))[:count])
            blocks[b, h, :len(at)] = at
    _check(c, _queries(g, 4, Hq, d, "f16", 1.5), [1] * 4, blocks=blocks)


@pytest.mark.parametrize("S,L,rows", [(1, 4999, 1), (1, 40000, 1), (2, 9000, 20), (40, 500, 1), (90, 300, 3)])
def test_work_that_is_shared_out(S, L, rows):
    g = np.random.default_rng([44, S, L])
    Hq, Hkv, d = 8, 2, 64
    lengths = [L] + [int(n) for n in g.integers(L // 2, L + 1, S - 1)]
    c = ch.filled(g, lengths, Hkv, d, 64, "i8")
    _check(c, _queries(g, S * rows, Hq, d, "f16", 4.0), [rows] * S)


@pytest.mark.parametrize("format", ["i8", "e4m3"])
@pytest.mark.parametrize("rows", [1, 9])
def test_scores_that_rise_and_scales_that_differ(rows, format):
    """Scales of values that span 2^40, and keys in the direction of the queries that grow all the way: levels are set again and again."""
    g = np.random.default_rng([45, rows])
    Hq, Hkv, d, L, page = 4, 2, 64, 777, 64
    c = ch.filled(g, [L, L], Hkv, d, page, format, dtype="bf16")
    c["vscale"] = np.where(np.isfinite(c["vscale"]), c["vscale"] * 2.0 ** g.integers(-20, 21, c["vscale"].shape), c["vscale"]).astype(np.float32)
    q = _queries(g, 2, Hq, d, "bf16", 6.0).repeat(rows, 0)
    q[:, 1::2] = q[:, ::2]
    code, _ = co.encode(q[rows, ::2].astype(np.float32), format)
    for n in range(L):                                       # the second sequence's scores rise from 0 to some hundreds
        i, at = c["table"][1, n // page], n % page
        c["k"][i, :, at], c["kscale"][i, :, at] = code, (0.002 if format == "i8" else 0.0006) * (1 + n) / 8
    _check(c, q, [rows, rows], "bf16", scale=0.125)
