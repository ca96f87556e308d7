"""How large calls on the paged cache may be, and what workspaces they ask for; nothing is launched."""
import pytest

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
