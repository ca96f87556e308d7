"""Copies of pages at the border of what one launch counts (2^32 threads, two stretches of 4 KiB to a workgroup of 256), without a GPU: refused calls launch nothing."""
import pytest

from tests import test_cache_pages as tp

cache = tp.cache

# sizes of a page and how many stretches it has: codes and scales of keys and values, and means
PAGES = [(dict(Hkv=1, d=64, page=16, kmean=None), 4), (dict(Hkv=9, d=64, page=16, kmean=None), 8), (dict(Hkv=14, d=64, page=64), 31), (dict(Hkv=1, d=64, page=16), 5)]


@pytest.mark.parametrize("kw,chunks", PAGES)
def test_copies_of_as_many_threads_as_no_launch_counts(kw, chunks):
    c = cache(**kw)
    for all in (1 << 25, (1 << 25) - 1):
        if all % chunks == 0:
            assert tp.copy(c, n=all // chunks) == 2
    assert tp.copy(c, n=(1 << 25) // chunks + 1) == 2


def test_room_with_copies_of_as_many_threads_as_no_launch_counts():
    """Refused before anything is planned: tables would name pages whose older tokens were never copied."""
    kw, chunks = PAGES[1]
    S = (1 << 25) // chunks
    assert tp.room(cache(S=S, table_width=4, **kw)) == 2
    assert tp.room(cache(S=S - 1, table_width=4, **kw)) == 4             # as far as the workspace, which is too small
