"""The oracle of the paged cache against what its definitions say, by hand."""
import numpy as np
import pytest

from oracle import cache_oracle as co
from tests import cache_harness as ch


def test_e4m3_values():
    t = co.E4M3
    assert t[0] == 0 and t[1] == 2.0 ** -9 and t[8] == 2.0 ** -6 and t[0x38] == 1.0 and t[0x7E] == 448 and t[0xFE] == -448
    assert np.isnan(t[0x7F]) and np.isnan(t[0xFF]) and (np.diff(t[:127]) > 0).all()


def test_codes_are_the_nearest_and_ties_go_to_even():
    c, s = co.encode(np.array([[127.0, 0.5, 1.5, 2.5, -0.5, -1.5, 126.49, 0.0]], np.float32), "i8")
    assert s[0] == 1.0 and list(c[0].astype(int) - 128) == [127, 0, 2, 2, 0, -2, 126, 0]
    c, s = co.encode(np.array([[448.0, 17.0, 19.0, 2.0 ** -10, 3 * 2.0 ** -10, -424.0, 433.0, 0.0]], np.float32), "e4m3")
    assert s[0] == 1.0 and list(co.E4M3[c[0]]) == [448, 16, 20, 0, 2.0 ** -8, -416, 448, 0]
    c, s = co.encode(np.array([[0.0, 0.0], [np.inf, 1.0], [2.0 ** -101, 0.0]], np.float32), "i8")
    assert s[0] == 1 and np.isnan(s[1]) and s[2] == 1 and (c == 128).all()


@pytest.mark.parametrize("format,step", [("i8", 0.5 / 127), ("e4m3", 2.0 ** -4)])
def test_what_is_held_is_within_half_a_step(format, step):
    g = np.random.default_rng(0)
    x = ch.rounded(g.standard_normal((50, 64)), "f16")
    c, s = co.encode(x, format)
    off = np.abs(co.values(c, s, format) - x)
    top = np.abs(x).max(-1, keepdims=True)
    assert (off <= (step * top if format == "i8" else np.maximum(step * np.abs(x), 2.0 ** -10 / 448 * top)) * (1 + 1e-6)).all()


def test_attention_of_the_oracle_is_softmax():
    g = np.random.default_rng(1)
    c = ch.filled(g, [37, 5], 2, 64, 16, "i8", shift=True)
    q = g.standard_normal((4, 4, 64))
    o, wide, _ = co.attend(c, q, ch.starts([3, 1]), 0.125)
    k, v = co.read({**c, "kshift": None}, None, 37)
    for t in range(3):
        s = k[0, 1, :35 + t] @ q[t, 2] * 0.125
        p = np.exp(s) / np.exp(s).sum()
        assert np.allclose(o[t, 2], p @ v[0, 1, :35 + t], rtol=1e-12)
    # a vector taken from all keys leaves the rows as they are
    k, _ = co.read(c, None, 37)
    s = k[0, 1, :37] @ q[2, 2] * 0.125
    p = np.exp(s - s.max())
    assert np.allclose(o[2, 2], p / p.sum() @ v[0, 1, :37], rtol=1e-9)
    tree = np.array([1, 3, 5, 1], np.uint64)
    o2, _, _ = co.attend(c, q, ch.starts([3, 1]), 0.125, tree=tree)
    assert np.allclose(o2[:2], o[:2]) and not np.allclose(o2[2], o[2])
    blocks = np.tile(np.array([0, 2, -1], np.int32), (2, 2, 1))
    o3, _, _ = co.attend(c, q, ch.starts([3, 1]), 0.125, blocks=blocks)
    at = list(range(16)) + list(range(32, 37))
    k, _ = co.read({**c, "kshift": None}, None, 37)
    s = k[0, 0, at] @ q[2, 1] * 0.125
    p = np.exp(s) / np.exp(s).sum()
    assert np.allclose(o3[2, 1], p @ v[0, 0, at], rtol=1e-12)
    picked = co.choose(c, q, ch.starts([3, 1]), 2, 1, 1)
    assert picked[0].tolist() == [[0, 2], [0, 2]] and picked[1].tolist() == [[0, -1], [0, -1]]
