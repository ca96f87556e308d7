"""CPU oracle of the paged 8-bit cache, from the definitions in include/pasa.h, in fp64 numpy.  Test infrastructure only.

A cache here is a dict of numpy arrays laid out like the library's: k, v uint8 [pages, Hkv, page, d]; kscale, vscale float32
[pages, Hkv, page]; kmean float32 [pages, Hkv, d] or None; kshift float32 [Hkv, d] or None; table int32 [S, W]; length int32 [S];
format "i8" or "e4m3".
"""
from __future__ import annotations

import numpy as np

E4M3 = np.array([np.nan if b & 127 == 127 else (-1.0) ** (b >> 7) * ((b & 7) / 8.0 * 2.0 ** -6 if b >> 3 & 15 == 0 else
                 (1 + (b & 7) / 8.0) * 2.0 ** ((b >> 3 & 15) - 7)) for b in range(256)])


def encode(x, format):
    """x float32 [..., d] -> codes uint8, scale float32.  Quotients are compared as exact fractions would be: fp64 holds the products."""
    x = np.asarray(x, np.float32).astype(np.float64)
    bad = ~np.isfinite(x).all(-1)
    x = np.where(bad[..., None], 0.0, x)
    top = np.abs(x).max(-1)
    scale = (top / (127.0 if format == "i8" else 448.0)).astype(np.float32)
    scale = np.where(top < 2.0 ** -100, np.float32(1), scale)
    s = scale.astype(np.float64)[..., None]
    q = x / s
    if format == "i8":
        n = np.floor(q)
        left = x - n * s                        # exact: n has 7 bits, s 24, x 24 and of the same size
        up = (left > s / 2) | ((left == s / 2) & (n % 2 == 1))
        codes = (np.clip(n + up, -127, 127) + 128).astype(np.uint8)
    else:
        grid = E4M3[:127]                       # 0 .. 448, ascending with the code
        a = np.abs(x)
        low = np.clip(np.searchsorted(grid, np.abs(q), side="right") - 1, 0, 126)
        high = np.minimum(low + 1, 126)
        middle = (grid[low] + grid[high]) / 2 * s
        up = (a > middle) | ((a == middle) & (low % 2 == 1))
        codes = (np.where(up, high, low) | np.where(np.signbit(x), 128, 0)).astype(np.uint8)
    return codes, np.where(bad, np.float32(np.nan), scale)


def values(codes, scale, format):
    x = codes.astype(np.float64) - 128.0 if format == "i8" else E4M3[codes]
    return x * scale.astype(np.float64)[..., None]


def _spans(c, row_start, R):
    """(sequence, tokens, first row, rows) as the library takes them."""
    page = c["k"].shape[2]
    for b in range(len(c["length"])):
        n = int(np.clip(c["length"][b], 0, c["table"].shape[1] * page))
        r0, r1 = (int(np.clip(row_start[b + i], 0, R)) for i in (0, 1))
        yield b, n, r0, max(0, r1 - r0)


def _page(c, b, place):
    i = int(c["table"][b, place])
    return i if 0 <= i < c["k"].shape[0] else None


def write(c, k, v, row_start):
    """Tokens enter; c is changed.  k, v float32 [R, Hkv, d]."""
    page = c["k"].shape[2]
    shift = 0 if c["kshift"] is None else c["kshift"]
    kc, ks = encode(np.float32(k) - np.float32(shift), c["format"])
    vc, vs = encode(v, c["format"])
    for b, n, r0, m in _spans(c, row_start, len(k)):
        touched = set()
        for t in range(m):
            pos = n - m + t
            if pos < 0:
                continue
            i = _page(c, b, pos // page)
            touched.add(pos // page)
            if i is not None:
                c["k"][i, :, pos % page], c["kscale"][i, :, pos % page] = kc[r0 + t], ks[r0 + t]
                c["v"][i, :, pos % page], c["vscale"][i, :, pos % page] = vc[r0 + t], vs[r0 + t]
        if c["kmean"] is not None:
            for p in touched:
                i = _page(c, b, p)
                if i is not None:
                    left = min(page, n - p * page)
                    c["kmean"][i] = values(c["k"][i, :, :left], c["kscale"][i, :, :left], c["format"]).mean(1).astype(np.float32)


def read(c, first, N):
    """k, v float64 [S, Hkv, N, d]."""
    P, Hkv, page, d = c["k"].shape
    S = len(c["length"])
    out = np.zeros((2, S, Hkv, N, d))
    for b, n, _, _ in _spans(c, np.zeros(S + 1, int), 0):
        for j in range(N):
            pos = int(first[b]) + j if first is not None else j
            i = _page(c, b, pos // page) if 0 <= pos < n else None
            if i is not None:
                out[0, b, :, j] = values(c["k"][i, :, pos % page], c["kscale"][i, :, pos % page], c["format"])
                if c["kshift"] is not None:
                    out[0, b, :, j] += c["kshift"]
                out[1, b, :, j] = values(c["v"][i, :, pos % page], c["vscale"][i, :, pos % page], c["format"])
    return out[0], out[1]


def choose(c, q, row_start, count, head, tail):
    """int32 [S, Hkv, count].  q float64 [R, Hq, d]."""
    P, Hkv, page, d = c["k"].shape
    G = q.shape[1] // Hkv
    out = np.full((len(c["length"]), Hkv, count), -1, np.int32)
    for b, n, r0, m in _spans(c, row_start, len(q)):
        pages = -(-n // page)
        if m == 0:
            continue
        for h in range(Hkv):
            rank = []
            for p in range(pages):
                i = _page(c, b, p)
                if p < head or p >= pages - tail:
                    key = (3, 0.0)
                elif i is None:
                    key = (-1, 0.0)
                else:
                    s = q[r0:r0 + m, h * G:(h + 1) * G].reshape(-1, d) @ c["kmean"][i, h].astype(np.float64)
                    key = (2, 0.0) if np.isnan(s).any() else (1, s.max())
                rank.append((-key[0], -key[1], p))
            at = sorted(p for _, _, p in sorted(rank)[:count])
            out[b, h, :len(at)] = at
    return out


def attend(c, q, row_start, scale, tree=None, blocks=None):
    """(o, sum of the weights times |v|, largest sum of |q_c k_c| of a seen key times scale) of every row and head, float64.
    q float64 [R, Hq, d]; rows that belong to no sequence are NaN."""
    P, Hkv, page, d = c["k"].shape
    R, Hq, _ = q.shape
    G = Hq // Hkv
    o, wide, size = np.full((R, Hq, d), np.nan), np.zeros((R, Hq, d)), np.zeros((R, Hq))
    for b, n, r0, m in _spans(c, row_start, R):
        for h in range(Hkv):
            places = range(-(-n // page)) if blocks is None else blocks[b, h]
            pos, k, v = [], [], []
            for p in places:
                i = _page(c, b, p) if 0 <= p < c["table"].shape[1] else None
                left = min(page, n - int(p) * page)
                if i is None or left <= 0:
                    continue
                pos += list(range(int(p) * page, int(p) * page + left))
                k.append(values(c["k"][i, h, :left], c["kscale"][i, h, :left], c["format"]))
                v.append(values(c["v"][i, h, :left], c["vscale"][i, h, :left], c["format"]))
            pos = np.array(pos, int)
            k, v = (np.concatenate(x) if x else np.zeros((0, d)) for x in (k, v))
            for t in range(m):
                nth = pos - (n - m)
                if tree is None:
                    see = nth <= t
                else:
                    bits = np.array([int(tree[r0 + t]) >> j & 1 for j in range(64)], bool)
                    see = (nth < 0) | ((nth < 64) & bits[np.clip(nth, 0, 63)])
                for g in range(h * G, (h + 1) * G):
                    with np.errstate(all="ignore"):
                        row = q[r0 + t, g]
                        s = (k[see] @ row) * scale
                        top = s.max() if len(s) else -np.inf
                        if not len(s) or top == -np.inf:
                            o[r0 + t, g] = 0.0
                            continue
                        p = np.exp(s - top)
                        p /= p.sum()
                        o[r0 + t, g] = p @ v[see]
                        wide[r0 + t, g] = p @ np.abs(v[see])
                        size[r0 + t, g] = (np.abs(k[see]) @ np.abs(row)).max() * scale
    return o, wide, size
