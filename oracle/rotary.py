"""Oracle: rotary positions and their frequencies.

Test infrastructure only (see the package docstring).  Pairs of a head's first ``dim`` values turn by
position * frequency; angles in extended precision.
"""
from __future__ import annotations

import math

import numpy as np

HALF, INTERLEAVED = "half", "interleaved"


def frequencies(dim, base, scaling, factor=1.0, original=0.0, low=0.0, high=0.0):
    if scaling == "base":
        base = base * factor ** (dim / (dim - 2))
    f = [base ** (-2 * i / dim) for i in range(dim // 2)]
    if scaling == "linear":
        return np.array([x / factor for x in f])
    out = []
    for i, x in enumerate(f):
        r = 1.0
        if scaling == "turns":
            r = min(max((original * x / (2 * math.pi) - low) / (high - low), 0.0), 1.0)
        if scaling == "index":
            i0, i1 = (dim * math.log(original / (2 * math.pi * n)) / (2 * math.log(base)) for n in (high, low))
            i0, i1 = max(math.floor(i0), 0), min(math.ceil(i1), dim - 1)
            r = min(max(1 - (i - i0) / max(i1 - i0, 0.001), 0.0), 1.0)
        out.append(x * (1 - r) / factor + x * r)
    return np.array(out)


def pair(i, dim, layout):
    return (i, i + dim // 2) if layout == HALF else (2 * i, 2 * i + 1)


def turn(x, positions, freq, amplitude, layout):
    """x [T, heads, hd] float64 at positions [T].  Returns (y, size) with size = |amplitude| (|a| + |b|) of each
    turned value, 0 of the others."""
    y, size = np.array(x, np.float64), np.zeros(x.shape)
    dim = 2 * len(freq)
    for t, p in enumerate(positions):
        for i, f in enumerate(freq):
            angle = np.longdouble(int(p)) * np.longdouble(f)
            c, s = (amplitude * float(fn(np.fmod(angle, 2 * np.arccos(np.longdouble(-1))))) for fn in (np.cos, np.sin))
            a, b = pair(i, dim, layout)
            y[t, :, a] = x[t, :, a] * c - x[t, :, b] * s
            y[t, :, b] = x[t, :, a] * s + x[t, :, b] * c
            size[t, :, a] = size[t, :, b] = abs(amplitude) * (np.abs(x[t, :, a]) + np.abs(x[t, :, b]))
    return y, size
