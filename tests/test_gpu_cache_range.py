"""Attention over the paged cache where scores or values are far from ordinary sizes."""
import numpy as np
import pytest

from oracle import cache_oracle as co
from tests import cache_bounds as cb
from tests import cache_harness as ch

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("L", [40, 700, 5000])
@pytest.mark.parametrize("rows", [1, 20])
def test_scores_far_below_zero(L, rows):
    """Scores down to -10^36, all of them below -10^30: the largest takes all the weight."""
    g = np.random.default_rng([31, L])
    Hq, Hkv, d, page = 4, 2, 64, 64
    c = ch.filled(g, [L, L], Hkv, d, page, "i8", dtype="bf16")
    c["k"][:] = 128 + 127
    at = g.permutation(L - rows)
    for n in range(L - rows):
        for b in range(2):
            c["kscale"][c["table"][b, n // page], :, n % page] = 1e24 * (1 + at[n])
    for n in range(L - rows, L):
        for b in range(2):
            c["kscale"][c["table"][b, n // page], :, n % page] = 1e29
    q = np.full((2 * rows, Hq, d), -ch.rounded(60000.0, "f16").astype(np.float64))
    got = ch.run_attend(ch.OnGpu(c), q, ch.starts([rows, rows]), 0.125, "f16")
    n = int(np.argmin(at))
    for b in range(2):
        i = c["table"][b, n // page]
        v = co.values(c["v"][i, :, n % page], c["vscale"][i, :, n % page], "i8").repeat(2, 0)
        # one weight: a rounding each of the scale's logarithm, reciprocal and quotient, and of the output
        assert (np.abs(got[rows * b:rows * (b + 1)] - v) <= (2.0 ** -11 + 2.0 ** -20) * np.abs(v) + 2.0 ** -25).all()


@pytest.mark.parametrize("format", ["i8", "e4m3"])
@pytest.mark.parametrize("exponent", [-99, -60, 0, 60, 126])
@pytest.mark.parametrize("L,rows", [(3000, 1), (900, 20), (262144, 1)])
def test_values_of_every_size_that_bf16_has(L, rows, exponent, format):
    """All values small or all large, weights nearly equal; half of the tokens as far above the others as a level allows."""
    g = np.random.default_rng([32, L, exponent + 200])
    Hq, Hkv, d, page = 2, 1, 64, 128
    c = ch.empty(g, 1, Hkv, d, page, -(-L // page), format, spare=0)
    c["length"][:] = L
    k = np.zeros((L, Hkv, d))
    k[np.arange(L) // 64 // 8 % 2 == 1, :, 0] = 7.75 * np.log(2.0) / 0.125      # P from 2^7 to 2^14.75
    v = 2.0 ** exponent * (1 + 0.1 * g.standard_normal((L, Hkv, d)))
    v[:, :, 5] *= g.choice([-1.0, 1.0], (L, Hkv))
    co.write(c, ch.rounded(k, "bf16"), ch.rounded(v, "bf16"), np.array([0, L], np.int32))
    q = np.zeros((rows, Hq, d))
    q[:, :, 0], q[:, 1, 1] = 1.0, 1.0
    got = ch.run_attend(ch.OnGpu(c), q, ch.starts([rows]), 0.125, "bf16")
    cb.check(got, cb.attend(c, q, ch.starts([rows]), 0.125, "bf16"))
