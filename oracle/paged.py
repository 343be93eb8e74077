"""The paged key/value cache of chunked generation: write, read, attention.

TEST INFRASTRUCTURE ONLY (see the package header).

An addition of this build, not of the paper: a clip generated chunk by chunk
keeps its earlier keys and values in pages of a shared pool.  The rows of the
int8 form are quantised head by head by the rule of cache.quantize_rows (fp32,
compared bit for bit); everything else is fp64.

Layouts: pages [n_pages, 2, H, page, d] (fp32 storage of bf16 values, or int8
codes), scale [n_pages, 2, H, page] fp32 or None, table [B, max_pages], lens [B],
row0 [B + 1]; row row0[b] + i of the call stands at position lens[b] - n_b + i.

Pins: a hand-worked two-page sequence; write then read gives the rounded values or
|v - q s| <= s (1/2 + 2^-14); attention against numpy's dense softmax on the rows in
order, over any page size; a permutation of the pages changes nothing; causal rows
equal the non-causal call of the shorter sequence; no key, no output.
"""
from __future__ import annotations

import numpy as np

from . import cache


def rows_of(lens, row0, max_pages, page):
    """(row, sequence, position) of every row at a position >= 0 that the table reaches."""
    out = []
    for b, n in enumerate(lens):
        for r in range(int(row0[b]), int(row0[b + 1])):
            p = int(n) - int(row0[b + 1]) + r
            if 0 <= p < max_pages * page:
                out.append((r, b, p))
    return out


def write(pages, scale, table, lens, row0, k, v):
    """The rows of k and v [n_rows, H d] (fp32) into the pages, in place; returns whether a
    quantised row was not finite."""
    H, page, d = pages.shape[2:]
    bad = False
    for r, b, p in rows_of(lens, row0, table.shape[1], page):
        pg, at = int(table[b, p // page]), p % page
        for i, src in enumerate((k, v)):
            x = np.asarray(src[r], dtype=np.float32)[:H * d].reshape(H, d)
            if scale is None:
                pages[pg, i, :, at] = cache.round_bf16(x)
            else:
                q, s, nf = cache.quantize_rows(x)
                pages[pg, i, :, at], scale[pg, i, :, at] = q, s
                bad |= bool(nf.any())
    return bad


def read(pages, scale, table, lens, row0, n_rows):
    """(k, v) [n_rows, H d] fp32: float(q) * s in one fp32 multiply, or the values."""
    H, page, d = pages.shape[2:]
    out = [np.zeros((n_rows, H * d), dtype=np.float32) for _ in range(2)]
    for r, b, p in rows_of(lens, row0, table.shape[1], page):
        pg, at = int(table[b, p // page]), p % page
        for i in range(2):
            x = pages[pg, i, :, at].astype(np.float32)
            if scale is not None:
                x = (x * scale[pg, i, :, at].astype(np.float32)[:, None]).astype(np.float32)
            out[i][r] = x.reshape(-1)
    return tuple(out)


def keys_values(pages, scale, table, n, b):
    """Keys and values [n, H, d] of sequence b in fp64."""
    H, page, d = pages.shape[2:]
    p = np.arange(n)
    pg, at = table[b, p // page], p % page
    kv = []
    for i in range(2):
        x = pages[pg, i, :, at].astype(np.float64)
        kv.append(x if scale is None else x * scale[pg, i, :, at].astype(np.float64)[..., None])
    return kv


def top_of(p, n, causal_block):
    """Keys that a row at position p of n sees."""
    if causal_block == 0:
        return n
    return 0 if p < 0 else min(n, (p // causal_block + 1) * causal_block)


def attend(pages, scale, table, lens, row0, q, Hq, causal_block=0):
    """(out, mass) [n_rows, Hq d] fp64: sum_j p_j v_j and sum_j p_j |v_j|, the size that
    errors of p and v are measured against; zeros for rows that see no key."""
    H, page, d = pages.shape[2:]
    q = np.asarray(q, dtype=np.float64)
    out = np.zeros((q.shape[0], Hq * d))
    mass = np.zeros_like(out)
    for b, n in enumerate(lens):
        n = int(n)
        kk, vv = keys_values(pages, scale, table, n, b)
        for r in range(int(row0[b]), int(row0[b + 1])):
            top = top_of(n - int(row0[b + 1]) + r, n, causal_block)
            if top == 0:
                continue
            for h in range(Hq):
                g, sl = h // (Hq // H), slice(h * d, (h + 1) * d)
                s = kk[:top, g] @ q[r, sl] / np.sqrt(d)
                p = np.exp(s - s.max())
                p /= p.sum()
                out[r, sl] = p @ vv[:top, g]
                mass[r, sl] = p @ np.abs(vv[:top, g])
    return out, mass
