"""Rotary positions without a GPU: frequencies, what the entry points refuse, the oracle's own properties."""
import ctypes
import math

import numpy as np
import pytest

import paper_2503_01873_amd as P
from oracle import rotary_oracle as ro
from tests import test_cache_refusals as refusals

SCALING = {"plain": P.ROTARY_PLAIN, "linear": P.ROTARY_LINEAR, "base": P.ROTARY_BASE, "ramp": P.ROTARY_RAMP, "waves": P.ROTARY_WAVES}
A = 1 << 20


@pytest.mark.parametrize("scaling", SCALING)
@pytest.mark.parametrize("rot,base,factor,original", [(128, 10000.0, 8.0, 4096), (64, 500000.0, 32.0, 8192), (2, 10000.0, 4.0, 2048), (20, 1e6, 1.0, 300),
                                                      (126, 10000.0, 2.5, 262144)])
def test_frequencies(scaling, rot, base, factor, original):
    r = P.pasa_rotary()
    fast = 4.0 if scaling == "waves" else 32.0
    P.pasa_rotary_set(r, P.ROTARY_PAIRS, rot, base, scaling=SCALING[scaling], factor=factor, original=original, slow=1.0, fast=fast, magnitude=1.5)
    want = ro.frequencies(rot, base, scaling, factor, original, 1.0, fast)
    assert np.allclose(np.array(r.freq[:rot // 2]), want, rtol=1e-13, atol=0)
    assert list(r.freq[rot // 2:]) == [0.0] * (64 - rot // 2)
    assert (r.magnitude, r.rot, r.layout) == (1.5, rot, P.ROTARY_PAIRS)
    if factor == 1.0:
        assert np.allclose(want, base ** (-np.arange(rot // 2) * 2 / rot), rtol=1e-13)
    if scaling == "base" and rot > 2:          # the slowest pair is slowed by the factor
        assert want[-1] * factor == pytest.approx(base ** (-(rot - 2) / rot), rel=1e-12) and want[0] == 1.0
    if scaling in ("ramp", "waves") and rot == 128:
        plain = base ** (-np.arange(64) * 2 / 128)
        assert want[0] == plain[0] and want[-1] == pytest.approx(plain[-1] / factor, rel=1e-13)
        assert ((want <= plain * (1 + 1e-13)) & (want >= plain / factor * (1 - 1e-13))).all() and (np.diff(want) < 0).all()


@pytest.mark.parametrize("kw,status", [
    (dict(rotary=None), 1), (dict(layout=2), 1), (dict(layout=-1), 1), (dict(rot=0), 1), (dict(rot=7), 1), (dict(rot=-2), 1), (dict(rot=130), 2), (dict(base=1.0), 1),
    (dict(base=math.nan), 1), (dict(base=math.inf), 1), (dict(scaling=5), 1), (dict(scaling=-1), 1), (dict(magnitude=math.inf), 1),
    (dict(scaling=P.ROTARY_LINEAR, factor=0.5), 1), (dict(scaling=P.ROTARY_BASE, factor=math.nan), 1), (dict(scaling=P.ROTARY_RAMP, factor=2.0), 1),
    (dict(scaling=P.ROTARY_RAMP, factor=2.0, original=4096, slow=4.0, fast=4.0), 1), (dict(scaling=P.ROTARY_WAVES, factor=2.0, original=4096, slow=0.0), 1),
    (dict(scaling=P.ROTARY_WAVES, factor=2.0, original=-1.0), 1), (dict(factor=math.nan), 0),
])
def test_settings_that_are_refused(kw, status):
    a = dict(rotary=P.pasa_rotary(), layout=0, rot=64, base=1e4, check=False)
    assert P.pasa_rotary_set(**{**a, **kw}) == status


def _rotary(rot=64, layout=0, **kw):
    """By hand: the library is not loaded while tests are collected (torch's HIP runtime has to come first where there is a GPU)."""
    r = P.pasa_rotary(magnitude=1.0, rot=rot, layout=layout)
    for i in range(rot // 2):
        r.freq[i] = 1e4 ** (-2 * i / rot)
    for n, x in kw.items():
        setattr(r, n, x)
    return r


def _bad_layout():
    r = _rotary()
    r.layout = 3
    return r


def _too_long():
    r = _rotary(rot=128)
    r.rot = 256                                                           # more pairs than there are frequencies
    return r


def _bad_frequency():
    r = _rotary()
    r.freq[31] = math.inf
    return r


@pytest.mark.parametrize("kw,status", [
    (dict(rotary=None), 1), (dict(x=None), 1), (dict(y=0), 1), (dict(x=A + 8), 1), (dict(y=2 * A + 2), 1), (dict(positions=3 * A + 2), 1),
    (dict(B=0), 1), (dict(H=-1), 1), (dict(N=0), 1), (dict(d=0), 1), (dict(d=96), 2), (dict(d=256), 2), (dict(io_dtype=2), 1), (dict(transposed=2), 1),
    (dict(rotary=_rotary(rot=128)), 1), (dict(rotary=_rotary(layout=0, rot=64), d=63), 1), (dict(rotary=_bad_layout()), 1),
    (dict(rotary=_rotary(magnitude=math.nan)), 1), (dict(rotary=_bad_frequency()), 1),
    (dict(x_strides=(8, 8, 4)), 1), (dict(x_strides=(-8, 8, 8)), 1), (dict(y_strides=(1000, 64, 56)), 1), (dict(y_strides=(1000, 0, 64)), 1),
    (dict(rotary=_too_long(), d=256), 1), (dict(H=0x7FFFFFFF, N=1, B=1), 2), (dict(H=(1 << 24) + 1, N=1, B=1), 2),
    (dict(y=A, x_strides=(640, 64, 128)), 1), (dict(row0=0x7FFFFFFF), 1), (dict(B=1 << 16, N=1 << 15), 2), (dict(H=1 << 20, N=1 << 20), 2),
])
def test_calls_that_are_refused(kw, status):
    a = dict(rotary=_rotary(), x=A, y=2 * A, B=2, H=2, N=5, d=64, check=False)
    assert P.pasa_rotate(**{**a, **kw}) == status


@pytest.mark.parametrize("kw,status", [
    (dict(cache=None), 1), (dict(cache=refusals.cache(d=96)), 2), (dict(cache=refusals.cache(length=None)), 1), (dict(rotary=None), 1), (dict(x=None), 1),
    (dict(y=2 * A + 8), 1), (dict(row_start=None), 1), (dict(row_start=3 * A + 1), 1), (dict(tree=4 * A + 4), 1), (dict(heads=0), 1), (dict(R=0), 1),
    (dict(x_stride=127), 1), (dict(x_stride=120), 1), (dict(y_stride=132), 1), (dict(y=A, y_stride=256), 1), (dict(rotary=_rotary(rot=66)), 1),
    (dict(io_dtype=-1), 1), (dict(transposed=-1), 1), (dict(R=0x7FFFFFFF), 2), (dict(cache=refusals.cache(S=0x7FFFFFFF, Hkv=1)), 2), (dict(heads=(1 << 24) + 1, x_stride=1 << 40, y_stride=1 << 40), 2), (dict(heads=1 << 24, x_stride=1 << 30, y_stride=1 << 30, R=1 << 26), 2),
])
def test_steps_that_are_refused(kw, status):
    a = dict(cache=refusals.cache(), rotary=_rotary(), x=A, y=2 * A, heads=2, R=3, x_stride=128, y_stride=128, row_start=3 * A, check=False)
    assert P.pasa_cache_rotate(**{**a, **kw}) == status


def test_strides_are_three():
    with pytest.raises(ValueError):
        P.pasa_rotate(_rotary(), A, 2 * A, 1, 1, 1, 64, x_strides=(1, 2))
    with pytest.raises(P.PasaError, match="pasa_rotate:"):
        P.pasa_rotate(None, A, 2 * A, 1, 1, 1, 64)
    with pytest.raises(P.PasaError, match="pasa_rotary_set:"):
        P.pasa_rotary_set(P.pasa_rotary(), 0, 3, 1e4)


def test_the_description_is_laid_out_as_in_c():
    r = _rotary(rot=64, layout=1, magnitude=2.0)
    assert ctypes.sizeof(r) == 64 * 8 + 8 + 8
    assert (ctypes.c_double * 65).from_address(r.data_ptr())[64] == 2.0
    assert list((ctypes.c_int * 2).from_address(r.data_ptr() + 520)) == [64, 1]


@pytest.mark.parametrize("pairs", [False, True])
def test_the_oracle_turns(pairs):
    """Products of queries and keys depend on the distance of their positions; turning back undoes; the transposed map is the gradient's."""
    g = np.random.default_rng(1)
    f = ro.frequencies(32, 1e4)
    q, k, w = (g.standard_normal((1, 1, 64)) for _ in range(3))
    at = lambda x, p, **kw: ro.rotate(x, np.array([p]), f, pairs, **kw)[0]
    a, b = (at(q, 100) * at(k, 40)).sum(), (at(q, 1060) * at(k, 1000)).sum()
    assert a == pytest.approx(b, rel=1e-10)
    assert np.allclose(at(at(q, 77), 77, transposed=True), q, atol=1e-13)
    assert (at(q, 9, magnitude=1.3) * w).sum() == pytest.approx((q * at(w, 9, magnitude=1.3, transposed=True)).sum(), rel=1e-12)
    e, i = 1e-6, 5
    d = q.copy()
    d[0, 0, i] += e
    assert ((at(d, 9) - at(q, 9)) * w).sum() / e == pytest.approx(at(w, 9, transposed=True)[0, 0, i], rel=1e-6)
