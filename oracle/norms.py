"""The norms around a gated residual in fp64.

TEST INFRASTRUCTURE ONLY (see the package header).

An addition of this build, not of the paper (whose block norm has neither modulation nor
gate): h = alpha x + beta gate N_after(y), n = N_before(h) (1 + scale) + shift, with the layer
norm, the norm by the root of the mean square, or none.

Pins: hand-worked rows; the layer norm without affine is block.layer_norm; mean 0 and
variance 1; gate 0 leaves x alone.
"""
from __future__ import annotations

import numpy as np


def norm(v, kind, weight=None, bias=None, eps=1e-6):
    v = np.asarray(v, dtype=np.float64)
    if kind == "none":
        return v
    if kind == "layer":
        v = v - v.mean(axis=1, keepdims=True)
    v = v / np.sqrt((v * v).mean(axis=1, keepdims=True) + eps)
    v = v if weight is None else v * np.asarray(weight, dtype=np.float64)
    return v if bias is None else v + np.asarray(bias, dtype=np.float64)


def gated(x, y=None, gate=None, scale=None, shift=None, before="layer", weight=None, bias=None, after="none",
          after_weight=None, after_bias=None, alpha=1.0, beta=1.0, eps=1e-6):
    """(h, n); gate, scale and shift are rows' own."""
    h = alpha * np.asarray(x, dtype=np.float64)
    if y is not None:
        h = h + beta * norm(y, after, after_weight, after_bias, eps) * (1.0 if gate is None else np.asarray(gate, np.float64))
    n = norm(h, before, weight, bias, eps)
    if scale is not None:
        n = n * (1 + np.asarray(scale, np.float64))
    return h, n if shift is None else n + np.asarray(shift, np.float64)
