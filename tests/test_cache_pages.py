"""The calls that share, give out and pack the pages of a cache, without a GPU: what they refuse, and the oracle's own properties."""
import numpy as np
import pytest

import paper_2503_01873_amd as P
from oracle import pages_oracle as po
from tests import cache4_harness as h4
from tests import test_cache_refusals as refusals

A = refusals.A
cache = refusals.cache
REFS = 20 * A


def copy(c, **kw):
    return P.pasa_cache_copy(**{**dict(to=c, of=c, to_pages=21 * A, from_pages=22 * A, n=3, check=False), **kw})


def fork(c, **kw):
    return P.pasa_cache_fork(**{**dict(cache=c, refs=REFS, source=21 * A, workspace=22 * A, workspace_bytes=1, check=False), **kw})


def room(c, **kw):
    return P.pasa_cache_room(**{**dict(cache=c, refs=REFS, R=2, row_start=21 * A, lacking=22 * A, workspace=23 * A, workspace_bytes=1, check=False), **kw})


def compact(c, **kw):
    return P.pasa_cache_compact(**{**dict(cache=c, refs=REFS, used=21 * A, workspace=22 * A, workspace_bytes=1, check=False), **kw})


def free(c, refs=REFS + 8):
    return P.pasa_cache_free(c, refs, check=False)


CALLS = [("copy", lambda c: copy(c, n=0)), ("fork", fork), ("room", room), ("compact", compact), ("free", free)]


@pytest.mark.parametrize("name,call", CALLS)
@pytest.mark.parametrize("kw,status", [(dict(k=None), 1), (dict(table=None), 1), (dict(length=6 * A + 2), 1), (dict(S=0), 1), (dict(format=2), 1), (dict(page=24), 2),
                                       (dict(d=32), 2)])
def test_caches_that_are_refused(name, call, kw, status):
    assert call(cache(**kw)) == status
    for size in (P.pasa_cache_fork_workspace, P.pasa_cache_compact_workspace, lambda c: P.pasa_cache_room_workspace(c, 4)):
        assert size(cache(**kw)) == 0


@pytest.mark.parametrize("name,call", CALLS)
def test_no_cache_at_all(name, call):
    assert call(None) == 1


@pytest.mark.parametrize("name,call", [("copy", lambda c: copy(c)), ("fork", fork), ("room", room), ("compact", compact), ("free", lambda c: free(c, REFS))])
def test_sizes_that_are_refused(name, call):
    assert call(cache(pages=(1 << 30) + 1)) == 2 and call(cache(Hkv=1 << 19, S=1)) == 2
    if name != "copy":
        assert call(cache(S=1 << 20, Hkv=1, table_width=4096)) == 2


@pytest.mark.parametrize("kw,status", [
    (dict(to_pages=None), 1), (dict(from_pages=0), 1), (dict(to_pages=21 * A + 2), 1), (dict(n=0), 1), (dict(n=-4), 1), (dict(of=cache(Hkv=1)), 1),
    (dict(of=cache(d=128)), 1), (dict(of=cache(page=32)), 1), (dict(of=cache(format=P.CACHE_I4)), 1), (dict(of=cache(kmean=None)), 1), (dict(of=None), 1),
    (dict(n=1 << 30), 2), (dict(of=cache(pages=1 << 31)), 1), (dict(of=cache(pages=(1 << 30) + 1)), 2),
])
def test_copies_that_are_refused(kw, status):
    assert copy(cache(), **kw) == status


@pytest.mark.parametrize("call,kw,status", [
    (fork, dict(), 4), (fork, dict(refs=None), 1), (fork, dict(refs=REFS + 4), 1), (fork, dict(source=None), 1), (fork, dict(source=21 * A + 1), 1),
    (fork, dict(workspace=None, workspace_bytes=1 << 20), 4), (fork, dict(workspace=22 * A + 64, workspace_bytes=1 << 20), 4),
    (room, dict(), 4), (room, dict(refs=0), 1), (room, dict(R=0), 1), (room, dict(R=-1), 1), (room, dict(row_start=None), 1), (room, dict(row_start=21 * A + 2), 1),
    (room, dict(lacking=22 * A + 1), 1), (room, dict(lacking=None), 4), (room, dict(workspace=23 * A + 16, workspace_bytes=1 << 20), 4),
    (compact, dict(), 4), (compact, dict(refs=REFS + 8), 1), (compact, dict(used=21 * A + 2), 1), (compact, dict(used=None), 4),
])
def test_calls_that_are_refused(call, kw, status):
    assert call(cache(), **kw) == status


def test_workspaces():
    c = cache()                                                          # 2 sequences of 4 places, 8 pages
    assert P.pasa_cache_fork_workspace(c) == 256 and P.pasa_cache_fork_workspace(cache(table_width=4096)) == (2 * 4096 + 2) * 4 // 256 * 256 + 256
    assert P.pasa_cache_room_workspace(c, 2) == 256 and P.pasa_cache_room_workspace(c, 0) == 0
    for R in (1, 100, 1 << 20):                                          # no more pages are given out than there are, or than rows
        assert P.pasa_cache_room_workspace(cache(pages=1000), R) == -(-(7 + min(R, R // 64 + 4, 1000)) * 4 // 256) * 256
    assert P.pasa_cache_compact_workspace(c) == 256
    assert fork(c, workspace_bytes=255) == 4 and room(c, workspace_bytes=255) == 4 and compact(c, workspace_bytes=255) == 4


def test_copies_beyond_what_a_launch_counts_are_refused():
    # of this cache a page is 2 + 2 + 1 + 1 + 1 stretches of 4 KiB
    assert copy(cache(), n=(1 << 25) // 7 + 1) == 2
    assert room(cache(S=(1 << 25) // 7 + 1, Hkv=2), workspace_bytes=1 << 40) == 2
    assert compact(cache(pages=620_000_000)) == 2 and compact(cache(pages=600_000_000)) == 4


def test_errors_name_the_entry_point():
    for name, call in (("copy", lambda: copy(cache(), n=0, check=True)), ("fork", lambda: fork(cache(), check=True)), ("room", lambda: room(cache(), check=True)),
                       ("compact", lambda: compact(cache(), check=True)), ("free", lambda: P.pasa_cache_free(cache(), None))):
        with pytest.raises(P.PasaError, match="pasa_cache_" + name + ":"):
            call()


def test_the_oracle_keeps_count():
    """Whatever happens, refs are the tables' counts, no written place is shared, and a page's tokens stay with who holds them."""
    g = np.random.default_rng(1)
    page, S, width = 16, 6, 5
    c = h4.empty(g, S, 1, 64, page, width)
    for n in po.BUFFERS:
        c[n] = c[n][:22]                                                 # fewer than the tables could hold
    c["table"][:] = -1
    c["refs"] = np.zeros(c["k"].shape[0], np.int32)
    held = [[] for _ in range(S)]                                        # what was written, token by token
    stamp = 0
    for step in range(300):
        kind = g.integers(0, 4)
        if kind == 0:
            source = np.where(g.random(S) < 0.6, np.arange(S), g.integers(-1, S, S))
            po.fork(c, source)
            held = [list(held[x]) if x >= 0 else [] for x in source]
        elif kind == 1:
            po.compact(c)
        elif kind == 2:
            for b in range(S):
                c["length"][b] = max(0, c["length"][b] - g.integers(0, 20))
                held[b] = held[b][:c["length"][b]]
            po.free(c)
        else:
            n = [min(int(g.integers(0, 12)), width * page - len(held[b])) for b in range(S)]
            rows = np.concatenate([[0], np.cumsum(n)])
            c["length"] += np.array(n, np.int32)
            lacking = po.room(c, rows, int(rows[-1]))
            for b in range(S):
                for t in range(n[b]):
                    stamp += 1
                    i, at = c["table"][b, len(held[b]) // page], len(held[b]) % page
                    assert i < 0 or c["refs"][i] == 1
                    if i >= 0:
                        c["kscale"][i, 0, at] = stamp
                    held[b].append(stamp if i >= 0 else None)
            assert lacking == 0 or (c["refs"] == 0).sum() == 0
            if lacking:                                                  # those sequences end
                gone = np.array([b if None not in held[b] else -1 for b in range(S)])
                po.fork(c, gone)
                held = [held[b] if gone[b] == b else [] for b in range(S)]
        assert np.array_equal(c["refs"], po.counts(c))
        for b in range(S):
            assert c["length"][b] == len(held[b])
            assert [c["kscale"][c["table"][b, t // page], 0, t % page] for t in range(len(held[b]))] == held[b]
