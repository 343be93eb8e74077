"""Seeded cases of 4-bit pages, as kv_case's: host bytes and scales, their values for the
oracle, and the same on the GPU.  What no sequence may use holds codes with scales of NaN,
infinity and the largest number."""
from dataclasses import dataclass

import numpy as np

import kv_case
from oracle import int4 as I

F32 = np.float32


@dataclass
class Case(kv_case.Case):
    """pages: bytes uint8 [n_pages, 2, H, page, d / 2], scale fp32 storage of bf16."""

    @property
    def values(self):
        return I.values(self.pages, self.scale)

    def device(self, ec, max_rows=None):
        import torch
        cuda = lambda a: torch.from_numpy(np.array(a)).cuda()       # noqa: E731
        rows = np.diff(self.row0)
        return (ec.KVPool(cuda(self.pages), cuda(self.scale).to(torch.bfloat16)),
                ec.KVBatch(cuda(self.table), cuda(self.lens), cuda(self.row0), self.n_rows,
                           int(rows.max(initial=0)) if max_rows is None else max_rows))


def make(page, H, d, lens, rows, seed=0, spare=2, amplitude=1.0):
    assert np.frexp(amplitude)[0] == 0.5                # scales keep their 5 significant bits
    c = kv_case.make("int8", page, H, d, lens, rows, seed=seed, spare=spare)
    g = np.random.default_rng(seed + 1000)
    shape = c.pages.shape[:4]
    codes = g.integers(-7, 8, (*shape, d)).astype(np.int8)
    exp = g.integers(-2, 2, (*shape, d // 32)) - 2
    scale = (g.integers(16, 32, (*shape, d // 32)) / 16 * 2.0 ** exp * amplitude).astype(F32)
    unused = np.isnan(c.scale)
    scale[unused] = g.choice(np.array([np.nan, np.inf, 31 * 2.0 ** 121], dtype=F32), (int(unused.sum()), d // 32))
    return Case(I.pack(codes), scale, c.table, c.lens, c.row0, H, d, page)
