"""Rotary positions in fp64, column by column.

TEST INFRASTRUCTURE ONLY (see the package header).

An addition of this build, not of the paper.  Pair i of n on an axis turns by p theta^(-i / n),
slowed down by one of the scalings (linear, ntk, or yarn's "NTK by parts", arXiv 2309.00071).

Pins: a quarter turn by hand; position 0 changes nothing; the inverse is the transposed map;
products of two turned vectors depend on the distance of their positions alone.
"""
from __future__ import annotations

import math

import numpy as np


def frequencies(axis_pairs, theta, scaling="none", factor=1.0, original=0.0, fast=32.0, slow=1.0):
    """(angles per position of every pair, factor of the turned columns)."""
    out = []
    for n in axis_pairs:
        base = theta * factor ** (n / (n - 1)) if scaling == "ntk" and n > 1 else theta
        for i in range(n):
            f = base ** (-i / n)
            if scaling == "linear":
                f /= factor
            if scaling == "yarn":
                turns = original / (2 * math.pi / f)          # within the context before scaling
                if turns <= slow:
                    f /= factor
                elif turns < fast:
                    part = (turns - slow) / (fast - slow)
                    f = (1 - part) * f / factor + part * f
            out.append(f)
    return np.array(out), 0.1 * math.log(factor) + 1 if scaling == "yarn" else 1.0


def turn(x, pos, d, axis_pairs, freq, size=1.0, layout="pairs", inverse=False, frame=None):
    """x [n, heads d] -> (fp64 result, the sizes |x1| + |x2| that errors are measured against)."""
    x = np.asarray(x, dtype=np.float64).reshape(len(x), -1, d)
    y, mass = x.copy(), np.zeros_like(x)
    pos = np.asarray(pos)
    if frame:
        pos = np.stack([pos // frame[0], pos % frame[0] // frame[1], pos % frame[1]], axis=1)
    pos = pos.reshape(len(x), -1)
    axis = np.repeat(np.arange(len(axis_pairs)), axis_pairs)
    n = sum(axis_pairs)
    for i in range(n):
        a, b = (2 * i, 2 * i + 1) if layout == "pairs" else (i, i + n)
        angle = pos[:, axis[i]].astype(np.float64) * freq[i] * (-1 if inverse else 1)
        c, s = size * np.cos(angle)[:, None], size * np.sin(angle)[:, None]
        y[:, :, a] = x[:, :, a] * c - x[:, :, b] * s
        y[:, :, b] = x[:, :, b] * c + x[:, :, a] * s
        mass[:, :, a] = mass[:, :, b] = abs(size) * (np.abs(x[:, :, a]) + np.abs(x[:, :, b]))
    return y.reshape(len(x), -1), mass.reshape(len(x), -1)
