"""pasa_cache_choose where scores are nearly equal: some are equal to others, some a few steps of 64 bits away from them."""
import numpy as np
import pytest

import paper_2503_01873_amd as P
from oracle import cache_oracle as co
from tests import cache_harness as ch

pytestmark = pytest.mark.gpu

STEP = 2.0 ** -52                        # of a score from 1 to 2 in 64 bits
D, HKV, PAGE, S = 64, 2, 16, 4


def _scores(g, width, far):
    """Two channels of the mean keys, exact in fp32, whose sum is the score: 1 + j steps for small j, many of them equal, one page 1 + 2^(far - 20)."""
    j = np.where(g.random(width) < 0.5, 2 ** g.integers(0, 10, width), g.integers(0, 2 ** g.integers(1, 10), width))
    j[g.random(width) < 0.3] = g.choice(j)
    one = np.ones(width)
    if far >= 0:
        one[g.integers(width)] += 2.0 ** (far - 20)
    return one, j * STEP


def _choose(c, q, count, head, tail):
    import torch
    gpu = ch.OnGpu(c)
    ws = torch.full((P.pasa_cache_choose_workspace(gpu.cache),), 0xFF, dtype=torch.uint8, device="cuda:0")
    out = torch.full((S, HKV, count), -7, dtype=torch.int32, device="cuda:0")
    tq, st = ch.tensor(q, "f16")
    P.pasa_cache_choose(gpu.cache, tq, S, st, ch.ints(range(S + 1)), q.shape[1], out, count, head, tail, ws, ws.numel(), torch.cuda.current_stream())
    torch.cuda.synchronize()
    return out.cpu().numpy()


def _cache(g, width, far):
    c = ch.empty(g, 1, HKV, D, PAGE, width, "i8", spare=0)
    c["kmean"][:] = 0.0
    for h in range(HKV):
        c["kmean"][:, h, 0], c["kmean"][:, h, 1] = _scores(g, width, far)
    c["table"] = np.stack([g.permutation(width) for _ in range(S)]).astype(np.int32)
    c["length"] = np.array([width * PAGE - int(x) for x in g.integers(0, PAGE, S)], np.int32)
    q = np.zeros((S, HKV, D))
    q[:, :, 0], q[:, :, 1] = 1.0, [[1.0], [2.0], [-1.0], [1.0]]          # sums stay below 2 by far: exact
    q[2, :, 0], q[3, 1, :2] = -1.0, -1.0
    return c, q


@pytest.mark.parametrize("far", range(-1, 20))
def test_every_place_of_the_first_digit(far):
    """The bit from which scores differ moves through a digit and more."""
    g = np.random.default_rng([21, far + 1])
    c, q = _cache(g, 40, far)
    for count in (1, 2, 3, 5, 8, 13, 20, 30, 39):
        assert np.array_equal(_choose(c, q, count, 0, 1), co.choose(c, q, ch.starts([1] * S), count, 0, 1)), count


@pytest.mark.parametrize("far", [-1, 0, 3, 13])
@pytest.mark.parametrize("width", [1024, 1025, 4097])
def test_every_size_of_the_table(width, far):
    g = np.random.default_rng([22, width, far + 1])
    c, q = _cache(g, width, far)
    for count in (7, width // 8, width // 2, width - 3):
        assert np.array_equal(_choose(c, q, count, 1, 1), co.choose(c, q, ch.starts([1] * S), count, 1, 1)), count


def test_three_scores_at_the_border():
    """One score a few steps above two that are equal, of which the first is the last one that is taken."""
    g = np.random.default_rng(23)
    c, q = _cache(g, 6, -1)
    q[:] = 0.0
    q[:, :, :2] = 1.0
    c["length"][:] = 6 * PAGE
    c["table"][:] = np.arange(6)
    for steps in [2 ** e for e in range(9)] + [3, 64 + 32, 128 + 7, 255]:
        c["kmean"][:, :, 0] = np.array([0, 5, 1, 1, 1, 0.5])[:, None]
        c["kmean"][:, :, 1] = np.array([0, 0, steps, 0, 0, 0])[:, None] * STEP
        assert np.array_equal(_choose(c, q, 4, 1, 0), np.broadcast_to([0, 1, 2, 3], (S, HKV, 4))), steps


@pytest.mark.parametrize("width,count", [(1024, 100), (4096, 900), (4097, 7)])
def test_pages_that_sequences_share(width, count):
    """Fifty pages in places of a long table: every score comes many times."""
    g = np.random.default_rng([24, width])
    c = ch.empty(g, 1, HKV, D, PAGE, 50, "i8", spare=0)
    c["kmean"] = g.standard_normal(c["kmean"].shape).astype(np.float32)
    c["table"] = g.integers(0, 50, (S, width)).astype(np.int32)
    c["length"] = np.full(S, width * PAGE - 3, np.int32)
    q = ch.rounded(g.standard_normal((S, 2 * HKV, D)), "f16").astype(np.float64)
    assert np.array_equal(_choose(c, q, count, 1, 1), co.choose(c, q, ch.starts([1] * S), count, 1, 1))
