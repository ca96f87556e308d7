"""Tokens of the largest numbers of their type: they come back finite, and so does attention over them, whatever a code's or a weight's rounding adds."""
import numpy as np
import pytest

import paper_2503_01873_amd as P
from oracle import cache4_oracle as c4
from oracle import cache_oracle as co
from tests import cache4_harness as h4
from tests import cache_harness as ch

pytestmark = pytest.mark.gpu

MOST = {"f16": 65504.0, "bf16": 255 * 2.0 ** 120}
FORMATS = ["i8", "e4m3", "i4"]


def _empty(g, format, *size, **kw):
    return h4.empty(g, *size, **kw) if format == "i4" else ch.empty(g, *size, format, **kw)


def _write(c, k, v, rows):
    (c4 if c["format"] == "i4" else co).write(c, k, v, rows)


def _plain(c):
    return c4.plain(c) if c["format"] == "i4" else c


def _on_gpu(c):
    return h4.OnGpu(c) if c["format"] == "i4" else ch.OnGpu(c)


def _tokens(g, n, Hkv, d, dtype):
    """Largest magnitudes from the type's largest number down by a step or some; the others anything below."""
    steps = 11 if dtype == "f16" else 8
    x = g.uniform(-1, 1, (n, Hkv, d)) * MOST[dtype]
    x[..., 0] = MOST[dtype] * (1 - g.integers(0, 9, (n, Hkv)) * 2.0 ** -steps)
    x[..., d // 2 + 1] = -x[..., 0]
    x[0], x[1] = MOST[dtype], -MOST[dtype]
    return ch.rounded(x, dtype)


def _read(gpu, S, Hkv, N, d, dtype):
    import torch
    out = [torch.full((S, Hkv, N, d), float("nan"), dtype=torch.float16 if dtype == "f16" else torch.bfloat16, device="cuda:0") for _ in range(2)]
    P.pasa_cache_read(gpu.cache, out[0], out[1], None, N, torch.cuda.current_stream(), io_dtype=ch.IO[dtype])
    torch.cuda.synchronize()
    return [x.double().cpu().numpy() for x in out]


@pytest.mark.parametrize("dtype", ["f16", "bf16"])
@pytest.mark.parametrize("shift", [False, True])
@pytest.mark.parametrize("d,page", [(64, 16), (128, 64)])
@pytest.mark.parametrize("format", FORMATS)
def test_the_largest_tokens_come_back_finite(format, d, page, shift, dtype):
    g = np.random.default_rng([d, shift])
    n, Hkv = 200, 2
    c = _empty(g, format, 1, Hkv, d, page, -(-n // page), mean=False)
    if shift:                                                            # so that what is held is larger than the type's numbers, where the key's bias has the other sign
        c["kshift"] = (g.choice([-1.0, 1.0], (Hkv, d)) * (60000 if dtype == "f16" else 1e36)).astype(np.float32)
    c["length"][:] = n
    gpu = _on_gpu(c)
    k, v = _tokens(g, n, Hkv, d, dtype), _tokens(g, n, Hkv, d, dtype)
    _write(c, k, v, ch.starts([n]))
    tk, st = ch.tensor(k, dtype)
    tv, _ = ch.tensor(v, dtype)
    P.pasa_cache_write(gpu.cache, tk, tv, n, st, ch.ints([0, n]), None, io_dtype=ch.IO[dtype])
    beyond = 0
    for got, want in zip(_read(gpu, 1, Hkv, n, d, dtype), co.read(_plain(c), None, n)):
        beyond += (np.abs(want) > MOST[dtype]).sum()
        assert np.isfinite(got).all()
        # what is held, rounded to fp32 and to the type; the type's largest number where it is more
        want = np.clip(want, -MOST[dtype], MOST[dtype])
        assert not (np.abs(got - want) > ch.HALF_STEP[dtype] * np.abs(want) * (1 + 2.0 ** -20) + 2.0 ** -24 * MOST[dtype] * 2).any()
    assert beyond > 0 or not (shift or (format == "i4" and dtype == "f16"))


@pytest.mark.parametrize("format", FORMATS)
def test_what_no_number_of_the_type_is_held_as_comes_back_infinite(format):
    """Written in bf16, read in fp16: a million is not 65504."""
    g = np.random.default_rng(1)
    c = _empty(g, format, 1, 1, 64, 16, 2, mean=False)
    c["length"][:] = 20
    k, v = (ch.rounded(x, "bf16") for x in (np.full((20, 1, 64), -1e6), np.full((20, 1, 64), 1e6)))
    k[:, :, 3], v[:, :, 40] = 0.0, 0.0
    _write(c, k, v, ch.starts([20]))
    gpu = _on_gpu(c)
    k, v = _read(gpu, 1, 1, 20, 64, "f16")
    assert (np.delete(k, 3, 3) == -np.inf).all() and (np.delete(v, 40, 3) == np.inf).all() and not k[..., 3].any() and not v[..., 40].any()
    o = ch.run_attend(gpu, np.zeros((1, 2, 64)), [0, 1], 0.125, "f16")
    assert (np.delete(o, 40, 2) == np.inf).all() and not o[..., 40].any()


def _bound(c, q, row_start, scale, dtype, keys):
    if c["format"] == "i4":
        return h4.attend(c, q, row_start, scale, dtype)
    ref = co.attend(c, q, row_start, scale)
    return ref[0], ch.attend_bound(c, ref, dtype, keys)


@pytest.mark.parametrize("dtype", ["f16", "bf16"])
@pytest.mark.parametrize("L", [1, 64, 3000])
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("format", FORMATS)
def test_attention_over_the_largest_values_is_finite(format, d, L, dtype):
    """Long sequences are merged from parts."""
    g = np.random.default_rng([d, L])
    Hq, Hkv = 4, 2
    c = _empty(g, format, 1, Hkv, d, 64, -(-L // 64) + 20, mean=False)
    c["length"][:] = L
    k = ch.rounded(g.standard_normal((L, Hkv, d)), dtype)
    v = _tokens(g, max(L, 2), Hkv, d, dtype)[:L]
    v[:, 0, :8], v[:, 1, d - 8:] = MOST[dtype], -MOST[dtype]             # of all tokens, so that the output is such a number
    _write(c, k, v, ch.starts([L]))
    q = ch.rounded(g.standard_normal((1, Hq, d)), dtype).astype(np.float64)
    got = ch.run_attend(_on_gpu(c), q, [0, 1], float(np.float32(d ** -0.5)), dtype)
    o, bound = _bound(c, q, [0, 1], float(np.float32(d ** -0.5)), dtype, L)
    assert np.isfinite(got).all()
    assert not (np.abs(got - np.clip(o, -MOST[dtype], MOST[dtype])) > bound).any()


@pytest.mark.parametrize("format", FORMATS)
def test_weights_that_round_upwards_do_not_make_the_largest_values_infinite(format):
    """One key of weight 2^7 and 63 whose weights lie just above the middle between two fp16 numbers: rounded, they come to 1 + 2^-11.2 times their sum."""
    g = np.random.default_rng(3)
    d, L, Hq = 64, 64, 2
    c = _empty(g, format, 1, 1, d, 64, 1, mean=False)
    c["length"][:] = L
    k, v = np.zeros((L, 1, d), np.float32), np.full((L, 1, d), 65504, np.float32)
    k[1:, 0, 0] = -1.0
    v[:, 0, 1::2] *= -1
    _write(c, k, v, ch.starts([L]))
    q = np.zeros((1, Hq, d))
    q[..., 0] = 1.0
    held = co.read(_plain(c), None, 2)[0][0, 0, 1, 0]
    scale = float(np.float32(np.log(128 / 64.035) / -held))
    o, bound = _bound(c, q, [0, 1], scale, "f16", L)
    got = ch.run_attend(_on_gpu(c), q, [0, 1], scale, "f16")
    assert np.isfinite(got).all() and not (np.abs(got - np.clip(o, -65504, 65504)) > bound).any()
