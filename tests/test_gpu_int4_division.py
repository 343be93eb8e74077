"""Attention over 4-bit pages where its work is divided between CTAs in every way, and its
kernel of 256-key blocks, against the oracle in fp64 (tolerance of test_gpu_int4.py).

Heads of 64 with up to 8 packed rows take blocks of 256 keys where
sequences x heads x keys that a table row covers >= 2 SMs x 16 x 256; `wide` widens a case's
table to that.  The workspace holds NaN, so that a partial sum nobody stored shows.
"""
import numpy as np
import pytest

pytestmark = pytest.mark.gpu

import int4_case                                   # noqa: E402
import kv_case                                     # noqa: E402
from oracle import paged as P                      # noqa: E402

TOL = 2.15 * 2.0 ** -8
HEADS = pytest.mark.parametrize("d", [64, 128])
PAGES = pytest.mark.parametrize("page", [16, 32, 64, 128])


@pytest.fixture(scope="module")
def ec():
    import torch
    if not torch.cuda.is_available():
        pytest.skip("needs a GPU")
    from paper_2608_02474_gb300 import echocache
    return echocache


def sms():
    import torch
    return torch.cuda.get_device_properties(0).multi_processor_count


def bf(a):
    import torch
    return torch.from_numpy(np.ascontiguousarray(a)).to("cuda", torch.bfloat16)


def wide(ec, c, batch, max_rows):
    """The batch with a table as wide as the blocks of 256 keys ask for; its further entries are none."""
    import torch
    B = len(c.lens)
    width = -(-2 * sms() * 16 * 256 // (B * c.H * c.page))
    table = torch.full((B, max(width, c.table.shape[1])), -1, dtype=torch.int32, device="cuda")
    table[:, :c.table.shape[1]] = batch.table
    return ec.KVBatch(table, batch.lens, batch.row0, c.n_rows, max_rows)


def attend(ec, pool, batch, q, Hq, cb):
    import torch
    ws = torch.empty(ec.echo_kv_attention_workspace_size(pool, batch, Hq) // 4, device="cuda")
    ws.fill_(float("nan"))
    return ec.echo_kv_attention(pool, batch, q, causal_block=cb, workspace=ws).float().cpu().numpy()


@PAGES
@pytest.mark.parametrize("d,max_rows", [(64, 2), (64, 1000), (128, 2), (128, 1000)])
def test_tables_that_pass_31_bits(ec, page, d, max_rows):
    """A table of 2^31 positions, one page over and over: the longest sequence is taken as far
    as 31 bits go, and the one beside it is as ever.  2^31 - 255: the first length of which 256-key
    blocks, counted in 31 bits, would be negative."""
    import torch
    c = int4_case.make(page, 1, d, [200, page], [2, 1], seed=4)
    q = kv_case.queries(3, d, 4)
    want, mass = P.attend(c.values, None, c.table, c.lens, c.row0, q, 1, 1)
    pool, batch = c.device(ec)
    table = torch.full((2, 2 ** 31 // page), int(c.table[1, 0]), dtype=torch.int32, device="cuda")
    table[0, :batch.table.shape[1]] = batch.table[0]
    lengths = ((page, 0), (2 ** 31 - 256, 0), (2 ** 31 - 255, 0), (2 ** 31 - 128, 0), (2 ** 31 - 127, 8))
    for n, status in lengths if page in (16, 128) else lengths[::2]:
        lens = torch.tensor([200, n], dtype=torch.int32, device="cuda")
        out = attend(ec, pool, ec.KVBatch(table, lens, batch.row0, 3, max_rows), bf(q), 1, 1)
        assert ec.echo_get_device_error() == status and np.isfinite(out).all()
        rows = 3 if n == page else 2
        assert (np.abs(out - want)[:rows] <= TOL * mass[:rows] + 1e-30).all()
