"""Keys and values in 4 bits: codes, scales and the words that hold them.

TEST INFRASTRUCTURE ONLY (see the package header).

An addition of this build, not of the paper.  32 neighbouring values u of a head, taken in
bf16, share s = the least number of 5 significant bits at or above max |u| / 7 (2^-112 at
least); a code is the whole number nearest to u / s, halves away from zero.  A word of four
bytes holds 8 columns: column 2 i in bits 4 i and up, 2 i + 1 in bits 16 + 4 i and up, each
as code + 8.  Everything here is exact: fp64 holds the quotients' halves, and the scale is
found by comparing 7 s with max |u|.

Pins: hand-worked groups; |u - code s| <= s / 2; s is no larger than it has to be; packing
and unpacking undo each other; every code s is a bf16 number.
"""
from __future__ import annotations

import numpy as np

from . import cache

LEAST = 2.0 ** -112


def scale_of(a: float) -> float:
    """The least m 2^e, 16 <= m <= 31 whole, with 7 m 2^e >= a."""
    if a <= 7 * LEAST:
        return LEAST
    e = int(np.floor(np.log2(a / 7))) - 4
    for exp in (e - 1, e, e + 1):
        for m in range(16, 32):
            if 7.0 * m * 2.0 ** exp >= a:
                return m * 2.0 ** exp
    raise AssertionError(a)


def quantize(x):
    """x [.., d] fp32 -> (codes int8 [.., d], scale fp32 [.., d / 32], not finite)."""
    u = cache.round_bf16(np.asarray(x, dtype=np.float32)).astype(np.float64)
    g = u.reshape(-1, 32)
    codes, scale = np.zeros(g.shape, dtype=np.int8), np.zeros(len(g), dtype=np.float32)
    bad = False
    for i, v in enumerate(g):
        a = np.abs(v).max()
        if not np.isfinite(a):
            scale[i], bad = a, True
            continue
        s = scale_of(a)
        scale[i] = s
        codes[i] = np.sign(v) * np.floor(np.abs(v) / s + 0.5)
    return codes.reshape(u.shape), scale.reshape(*u.shape[:-1], -1), bad


def pack(codes):
    """codes [.., d] -> bytes uint8 [.., d / 2]."""
    c = (np.asarray(codes).astype(np.int64) + 8).reshape(*codes.shape[:-1], -1, 8)
    word = sum(c[..., k] << (4 * (k // 2) + 16 * (k % 2)) for k in range(8)).astype("<u4")
    return word.view(np.uint8).reshape(*codes.shape[:-1], -1)


def unpack(pages):
    """bytes [.., d / 2] -> codes int8 [.., d]."""
    word = np.ascontiguousarray(pages).view("<u4").astype(np.int64)
    c = np.stack([(word >> (4 * (k // 2) + 16 * (k % 2))) % 16 - 8 for k in range(8)], axis=-1)
    return c.reshape(*pages.shape[:-1], -1).astype(np.int8)


def values(pages, scale):
    """What bytes [.., d / 2] and scales [.., d / 32] stand for, fp32 (exact)."""
    with np.errstate(invalid="ignore", over="ignore"):
        return unpack(pages).astype(np.float32) * np.repeat(np.asarray(scale, dtype=np.float32), 32, axis=-1)
