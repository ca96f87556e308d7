"""Copies between pools whose keys have something else taken off them, without a GPU: held keys would stand for others there."""
import pytest

from tests import test_cache_pages as tp

A, cache = tp.A, tp.cache


@pytest.mark.parametrize("to,of,status", [(None, 30 * A, 1), (30 * A, None, 1), (30 * A, 31 * A, 2), (30 * A, 30 * A, 2), (None, None, 2)])
def test_pools_of_which_one_has_a_shift(to, of, status):
    """Where both have one its values, which the host does not see, are the caller's; n is refused then, so that nothing is launched."""
    assert tp.copy(cache(kshift=to), of=cache(kshift=of), n=1 << 30) == status
