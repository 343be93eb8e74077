"""Seeded cases of the paged key/value cache: host arrays for the oracle, and the same on
the GPU.  What no sequence may use (pages of none, slots at and past a sequence's length)
holds NaN, or int8 codes with NaN scales."""
from dataclasses import dataclass

import numpy as np

from synth import generate as G

F32 = np.float32


@dataclass
class Case:
    pages: np.ndarray      # fp32 storage of bf16 values, or int8
    scale: np.ndarray      # fp32 or None
    table: np.ndarray
    lens: np.ndarray
    row0: np.ndarray
    H: int
    d: int
    page: int

    @property
    def n_rows(self):
        return int(self.row0[-1])

    def device(self, ec, max_rows=None):
        """(pool, batch) over copies on the GPU."""
        import torch
        cuda = lambda a: torch.from_numpy(np.array(a)).cuda()       # noqa: E731
        pages = cuda(self.pages)
        if self.scale is None:
            pages = pages.to(torch.bfloat16)
        rows = np.diff(self.row0)
        return (ec.KVPool(pages, None if self.scale is None else cuda(self.scale)),
                ec.KVBatch(cuda(self.table), cuda(self.lens), cuda(self.row0), self.n_rows,
                           int(rows.max(initial=0)) if max_rows is None else max_rows))


def make(form, page, H, d, lens, rows, seed=0, spare=2, amplitude=1.0):
    g = np.random.default_rng(seed)
    B = len(lens)
    need = [-(-n // page) for n in lens]
    n_pages = sum(need) + spare
    order = g.permutation(n_pages)
    table = np.full((B, max(max(need, default=0), 1)), -1, dtype=np.int32)
    at = 0
    for b, n in enumerate(need):
        table[b, :n] = order[at:at + n]
        at += n
    if form == "int8":
        pages = g.integers(-127, 128, (n_pages, 2, H, page, d)).astype(np.int8)
        scale = ((0.5 + g.random((n_pages, 2, H, page))) / 64 * amplitude).astype(F32)
        poison = scale
    else:
        x = g.standard_normal((n_pages, 2, H, page, d)).astype(F32) * F32(amplitude)
        pages, scale = G.to_bf16_values(x), None
        poison = pages
    free = order[at:]
    poison[free] = np.nan
    for b, n in enumerate(lens):
        if n % page:
            poison[table[b, n // page], :, :, n % page:] = np.nan
    row0 = np.concatenate([[0], np.cumsum(rows)]).astype(np.int32)
    return Case(pages, scale, table, np.array(lens, dtype=np.int32), row0, H, d, page)


def queries(n_rows, cols, seed, scale=1.0):
    return G.to_bf16_values(np.random.default_rng(seed + 77).standard_normal((n_rows, cols))
                            .astype(F32) * F32(scale))
