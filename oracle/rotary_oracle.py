"""CPU oracle of rotary positions, from the definitions in include/pasa.h, in fp64 numpy.  Test infrastructure only."""
from __future__ import annotations

import math

import numpy as np


def frequencies(rot, base, scaling="plain", factor=1.0, original=0.0, slow=1.0, fast=32.0):
    out = []
    if scaling == "base" and rot > 2:
        base = base * factor ** (rot / (rot - 2))
    for i in range(rot // 2):
        f = base ** (-2 * i / rot)
        if scaling == "linear":
            f /= factor
        if scaling in ("ramp", "waves"):
            if scaling == "waves":
                keep = (original * f / (2 * math.pi) - slow) / (fast - slow)
            else:
                first, last = (rot * math.log(original / (2 * math.pi * t)) / (2 * math.log(base)) for t in (fast, slow))
                first, last = max(0, math.floor(first)), min(rot - 1, math.ceil(last))
                keep = 1 - (i - first) / max(0.001, last - first)
            keep = min(1.0, max(0.0, keep))
            f = f / factor * (1 - keep) + f * keep
        out.append(f)
    return np.array(out)


def rotate(x, position, freq, pairs, magnitude=1.0, transposed=False):
    """x float64 [..., heads, d], position [...].  (y, sum of the magnitudes of an element's two products)"""
    angle = np.asarray(position, np.float64)[..., None, None] * freq
    c, s = magnitude * np.cos(angle), magnitude * np.sin(angle) * (-1 if transposed else 1)
    rot = 2 * len(freq)
    a, b = (slice(0, rot, 2), slice(1, rot, 2)) if pairs else (slice(0, rot // 2), slice(rot // 2, rot))
    y, wide = x.copy(), np.zeros_like(x)
    y[..., a], y[..., b] = x[..., a] * c - x[..., b] * s, x[..., a] * s + x[..., b] * c
    wide[..., a], wide[..., b] = np.abs(x[..., a] * c) + np.abs(x[..., b] * s), np.abs(x[..., a] * s) + np.abs(x[..., b] * c)
    return y, wide


def positions(length, row_start, R, most, tree=None):
    """Of every row of a step its position, None where it belongs to no sequence."""
    out = [None] * R
    for b in range(len(length)):
        n = int(np.clip(length[b], 0, most))
        r0, r1 = (int(np.clip(row_start[b + i], 0, R)) for i in (0, 1))
        m = max(0, r1 - r0)
        for t in range(m):
            depth = t if tree is None else sum(int(tree[r0 + t]) >> j & 1 for j in range(min(m, 64)) if j != t)
            out[r0 + t] = n - m + depth
    return out
