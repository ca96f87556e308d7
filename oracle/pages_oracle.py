"""CPU oracle of the calls that share, give out, take back and pack the pages of a cache, from the definitions in include/pasa.h, one entry after the other.
Test infrastructure only.

A cache is a dict as in cache_oracle (k, v, kscale, vscale, kmean or None, table, length) with refs int32 [pages]; all of them are changed.
"""
from __future__ import annotations

import numpy as np

BUFFERS = ("k", "v", "kscale", "vscale", "kmean")


def _pool(c):
    return len(c["refs"])


def _in(c, p):
    return 0 <= p < _pool(c)


def _page(c):
    return c["kscale"].shape[2]


def _length(c, b):
    return int(np.clip(c["length"][b], 0, c["table"].shape[1] * _page(c)))


def counts(c):
    """What refs have to be."""
    held = c["table"][(c["table"] >= 0) & (c["table"] < _pool(c))]
    return np.bincount(held, minlength=_pool(c)).astype(np.int32)


def copy(to, of, to_pages, from_pages):
    for p, q in zip(to_pages, from_pages):
        if 0 <= p < to["k"].shape[0] and 0 <= q < of["k"].shape[0]:
            for n in BUFFERS:
                if to.get(n) is not None:
                    to[n][p] = of[n][q]


def fork(c, source):
    table, length = c["table"].copy(), [_length(c, b) for b in range(len(c["length"]))]
    for b, x in enumerate(source):
        if x == b:
            continue
        for p in c["table"][b]:
            if _in(c, p):
                c["refs"][p] -= 1
        n = length[x] if 0 <= x < len(length) else 0
        places = -(-n // _page(c))
        c["table"][b] = -1
        if places:
            c["table"][b, :places] = table[x, :places]
        c["length"][b] = n
        for p in c["table"][b]:
            if _in(c, p):
                c["refs"][p] += 1


def free(c):
    for b in range(len(c["length"])):
        for i in range(-(-_length(c, b) // _page(c)), c["table"].shape[1]):
            if _in(c, c["table"][b, i]):
                c["refs"][c["table"][b, i]] -= 1
            c["table"][b, i] = -1


def room(c, row_start, R):
    """How many places are without a page."""
    page, lacking = _page(c), 0
    pages = [p for p in range(_pool(c)) if c["refs"][p] == 0]
    for b in range(len(c["length"])):
        n = _length(c, b)
        r0, r1 = (int(np.clip(row_start[b + i], 0, R)) for i in (0, 1))
        if r1 <= r0 or n == 0:
            continue
        first = max(0, n - (r1 - r0))
        for i in range(first // page, (n - 1) // page + 1):
            old = int(c["table"][b, i])
            if _in(c, old):
                if c["refs"][old] == 1:
                    continue
                c["refs"][old] -= 1
            new = pages.pop(0) if pages else -1
            c["table"][b, i] = new
            if new < 0:
                lacking += 1
                continue
            c["refs"][new] = 1
            if _in(c, old) and i * page < first:
                copy(c, c, [new], [old])
    return lacking


def compact(c):
    """Pages in use."""
    n = int((c["refs"] != 0).sum())
    to = [p for p in range(n) if c["refs"][p] == 0]
    of = [p for p in range(n, _pool(c)) if c["refs"][p] != 0]
    now = dict(zip(of, to))
    c["table"][:] = [[now.get(int(p), int(p)) for p in row] for row in c["table"]]
    copy(c, c, to, of)
    for p, q in zip(to, of):
        c["refs"][p], c["refs"][q] = c["refs"][q], 0
    return n
