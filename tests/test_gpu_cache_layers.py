"""Layers of a model: each has a pool, a table, lengths and counts, and gets every call; tables stay alike, and what each layer holds moves with its own."""
import numpy as np
import pytest

from oracle import pages_oracle as po
from tests import cache_harness as ch
from tests import pages_harness as ph

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("format", ["i8", "i4"])
def test_layers_with_a_table_each(format):
    g = np.random.default_rng(1)
    S, Hkv, d, page, width = 7, 2, 64, 16, 5
    layers = [ph.pool(g, S, Hkv, d, page, width, 60, format, mean=i == 0) for i in range(3)]
    ph.hold(g, layers[0], g.integers(1, (width - 2) * page, S), 0.3)
    for c in layers[1:]:
        for n in ("table", "length", "refs"):
            c[n] = layers[0][n].copy()
    on_gpu = [ph.OnGpu(c) for c in layers]
    assert not np.array_equal(layers[0]["k"], layers[1]["k"])
    moved = 0
    for turn in range(5):
        source, n = g.integers(-1 if turn == 3 else 0, S, S), g.integers(0, 6, S)
        lacking = []
        for c, gpu in zip(layers, on_gpu):
            before = c["k"].copy()
            po.fork(c, source)
            gpu.fork(source)
            m = np.minimum(n, width * page - c["length"])
            rows = ch.starts(m)
            c["length"] += m.astype(np.int32)
            gpu.t["length"].add_(ch.ints(m))
            lacking.append((po.room(c, rows, int(rows[-1]) + 1), gpu.room(rows, int(rows[-1]) + 1)))
            if turn % 2:
                po.compact(c)
                assert gpu.compact() == (c["refs"] != 0).sum()
            gpu.same(c)
            moved += (before != c["k"]).any()
        assert lacking == [(0, 0)] * 3
        for c in layers[1:]:
            assert all(np.array_equal(c[x], layers[0][x]) for x in ("table", "length", "refs"))
    assert moved >= 9                                                    # every layer's contents, in most turns
