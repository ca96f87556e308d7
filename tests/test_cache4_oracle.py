"""The oracle of the cache in 4 bits against the definition by fractions, and what its entry points refuse; nothing is launched."""
from fractions import Fraction

import numpy as np
import pytest

import paper_2503_01873_amd as P
from oracle import cache4_oracle as c4
from oracle import cache_oracle as co
from tests import cache4_harness as h4
from tests import cache_harness as ch
from tests import test_cache_refusals as refusals


def _nearest(x, unit):
    return round(Fraction(float(x)) / unit)                               # Python rounds fractions to the nearest, ties to even


@pytest.mark.parametrize("dtype", ["f16", "bf16", "f32"])
@pytest.mark.parametrize("d", [64, 128])
def test_codes_are_those_of_the_definition(d, dtype):
    g = np.random.default_rng(d)
    x = (g.standard_normal((40, d)) * 2.0 ** g.integers(-9, 9, (40, 1))).astype(np.float32)
    x[1], x[2, 5:], x[3] = 0.0, 0.0, 2.0 ** -99
    x[4, :32], x[5, 32:64] = 2.0 ** -20, 49.0                             # a group far below the others; 1568 = 49 * 32
    x[6] = g.integers(-14, 15, d) / 2.0                                   # ties
    if dtype != "f32":
        x = ch.rounded(x, dtype)
    codes, factors, scales = c4.encode(x)
    for row, code, factor, scale in zip(x, codes, factors, scales):
        top = Fraction(float(np.abs(row).max()))
        s = Fraction(float(scale))
        if top < Fraction(2) ** -98:
            assert s == 1 and (factor == 1).all() and not code.any()
            continue
        mantissa = s / Fraction(2) ** int(np.floor(np.log2(float(scale))))
        assert s * 1568 >= top and (mantissa * 128).denominator == 1
        assert (mantissa - Fraction(1, 128)) / mantissa * s * 1568 < top        # the next one below is too small
        for j in range(d // 32):
            part = row[32 * j:32 * j + 32]
            assert factor[j] == max(1, _nearest(np.abs(part).max(), 7 * s)) <= 224
            assert all(int(n) == max(-7, min(7, _nearest(y, s * int(factor[j])))) for n, y in zip(code[32 * j:32 * j + 32], part))


def test_numbers_are_held_exactly_by_fp16():
    n = np.arange(-7, 8)[:, None] * np.arange(1, 225)
    assert np.array_equal(n.astype(np.float16).astype(np.int64), n)
    # what is taken off: 72 * factor, and a code beside 64
    f = np.arange(1, 225)
    assert np.array_equal((72 * f).astype(np.float16).astype(np.int64), 72 * f)
    assert np.array_equal((np.arange(16) * 16 + 0x5400).astype(np.uint16).view(np.float16), 64 + np.arange(16))


def test_pages_hold_what_was_put_there():
    g = np.random.default_rng(3)
    c = h4.empty(g, 1, 2, 64, 16, 2)
    c["length"][:] = 20
    k, v = (ch.rounded(g.standard_normal((20, 2, 64)), "f16") for _ in range(2))
    c4.write(c, k, v, ch.starts([20]))
    assert c4.sizes(c) == (16, 64)
    back = co.read(c4.plain(c), None, 20)
    for x, y in ((k, back[0]), (v, back[1])):
        code, factor, scale = c4.encode(x)
        want = code * np.repeat(factor.astype(float), 32, -1) * scale[..., None].astype(float)
        assert np.array_equal(want, y[0].transpose(1, 0, 2))
        # half a step, or what the factor leaves beyond 7: at most half of a scale times 7
        assert (np.abs(want - x) <= np.maximum(0.5 * np.repeat(factor.astype(float), 32, -1), 3.5) * scale[..., None]).all()


I4 = dict(format=P.CACHE_I4)


@pytest.mark.parametrize("name,call", refusals.CALLS)
@pytest.mark.parametrize("kw,status", [
    (dict(k=None), 1), (dict(v=2 * refusals.A + 8), 1), (dict(kscale=None), 1), (dict(format=3), 1), (dict(format=5), 1), (dict(d=32), 2), (dict(page=8), 2),
    (dict(table_width=16385, page=16), 2),
])
def test_caches_that_are_refused(name, call, kw, status):
    assert call(refusals.cache(**{**I4, **kw})) == status


def test_calls_that_are_refused():
    c = refusals.cache(**I4)
    assert refusals.write(c, R=0) == 1 and refusals.read(c, N=0) == 1 and refusals.write(c, row_stride=120) == 1
    assert refusals.choose(c) == 4 and refusals.attend(c) == 4 and refusals.attend(c, Hq=3) == 1
    need = P.pasa_attn_cache_workspace(c, 2, 4)
    assert need == P.pasa_attn_cache_workspace(refusals.cache(), 2, 4) > 0
    assert refusals.attend(c, workspace_bytes=need - 1) == 4
