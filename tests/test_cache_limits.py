"""How large calls on the paged cache may be, and what workspaces they ask for; nothing is launched."""
import pytest

import paper_2503_01873_amd as P
from tests.test_cache_refusals import cache, choose, read, write


@pytest.mark.parametrize("call", [
    lambda: write(cache(), R=1 << 30),                                                   # 2^24 pages of 64 tokens, two heads
    lambda: write(cache(S=1 << 23), R=1 << 24),
    lambda: read(cache(S=1 << 13, Hkv=1), N=1 << 17),                                    # 2^11 stretches each
    lambda: read(cache(S=1 << 23), N=1),
    lambda: choose(cache(S=1 << 15, table_width=16384, page=16), workspace_bytes=1 << 60),
    lambda: choose(cache(S=1 << 21), count=4, workspace_bytes=1 << 60),
])
def test_launches_of_2_to_the_32_threads_are_refused(call):
    assert call() == 2


@pytest.mark.parametrize("Hkv,G", [(1, 1), (2, 4), (4, 7), (8, 1), (1, 20)])
@pytest.mark.parametrize("S", [1, 3, 16, 300])
def test_a_workspace_is_enough_for_fewer_rows(S, Hkv, G):
    for width in (1, 16, 17, 40, 128, 4096):
        c = cache(S=S, Hkv=Hkv, d=128, table_width=width)
        needs = [P.pasa_attn_cache_workspace(c, R, G * Hkv) for R in sorted({*range(1, 140), 16 * S // G, 16 * S // G + 1, 5000} - {0})]
        assert needs[0] > 0 and needs == sorted(needs), width
