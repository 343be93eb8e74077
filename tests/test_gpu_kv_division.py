"""Attention over the paged cache where every CTA takes whole items first and the rest is
divided, against the oracle in fp64 (tolerance of test_gpu_kv_attention.py: two roundings
to bf16, 2.15 * 2^-8 of sum_j p_j |v_j|).

The kernels for few rows run two CTAs per SM, those for chunks one; an item is a sequence,
a key/value head and a tile of rows.  Tables of more than 768 keys (chunks: 1024) are
divided.  The workspace holds NaN, so that a partial sum nobody stored shows.
"""
import numpy as np
import pytest

pytestmark = pytest.mark.gpu

import kv_case                                     # noqa: E402
from oracle import paged as P                      # noqa: E402

TOL = 2.15 * 2.0 ** -8


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


def check(ec, c, group, cb, max_rows=None):
    import torch
    Hq = c.H * group
    q = kv_case.queries(c.n_rows, Hq * c.d, 1, 1.5)
    want, mass = P.attend(c.pages, c.scale, c.table, c.lens, c.row0, q, Hq, cb)
    pool, batch = c.device(ec, max_rows)
    ws = torch.empty(ec.echo_kv_attention_workspace_size(pool, batch, Hq) // 4, device="cuda")
    ws.fill_(float("nan"))
    out = ec.echo_kv_attention(pool, batch, torch.from_numpy(q).to("cuda", torch.bfloat16), causal_block=cb,
                               workspace=ws).float().cpu().numpy()
    assert ec.echo_get_device_error() == 0
    bad = ~(np.abs(out - want) <= TOL * mass + 1e-30)
    assert not bad.any(), (int(bad.sum()), np.argwhere(bad.any(axis=1)).ravel()[:8].tolist())


FORMS = pytest.mark.parametrize("form", ["bf16", "int8"])
HEADS = pytest.mark.parametrize("d", [64, 128])


@FORMS
@HEADS
@pytest.mark.parametrize("chunks", [False, True])
@pytest.mark.parametrize("left", [1, 8])
def test_equal_items_and_a_few_more(ec, form, d, chunks, left):
    """One item for every CTA and a few over: CTAs get one unit of those, or none."""
    items = sms() * (1 if chunks else 2) + left
    H = max(h for h in range(1, 10) if items % h == 0)
    n = 1200 if chunks else 900
    c = kv_case.make(form, 128, H, d, [n] * (items // H), [1] * (items // H), seed=left)
    check(ec, c, 1, 1, 1000 if chunks else None)


@FORMS
@pytest.mark.parametrize("chunks", [False, True])
@pytest.mark.parametrize("seqs", [4, 50, 700])
def test_ragged_items_in_rounds(ec, form, chunks, seqs):
    """More than two items for every CTA, no more sequences than a block has warps, more
    than that, and more than it has threads."""
    g = np.random.default_rng(seqs)
    H = -(-int(2.3 * sms() * (1 if chunks else 2)) // seqs)
    lens = [int(n) for n in g.integers(700, 1100 if chunks else 900, seqs)]
    lens[seqs // 2] = 1100 if chunks else 900
    rows = [int(r) for r in g.integers(1, 4, seqs)]
    c = kv_case.make(form, 16, H, 64, lens, rows, seed=seqs)
    check(ec, c, 1, 1, 1000 if chunks else None)


@FORMS
@HEADS
def test_tiles_of_long_chunks_in_rounds(ec, form, d):
    """Several tiles of a sequence, which see more keys from tile to tile."""
    H = -(-sms() * 13 // 50)
    c = kv_case.make(form, 64, H, d, [1200, 1100], [600, 300], seed=2)
    check(ec, c, 1, 1)


@FORMS
@pytest.mark.parametrize("chunks", [False, True])
def test_items_without_keys_among_rounds(ec, form, chunks):
    """Sequences that are empty, short, or without rows between the others."""
    items = sms() * (1 if chunks else 2)
    H = 6
    lens, rows = [], []
    for i in range(items // H):
        lens += [1100 if i % 3 else 1090, 0 if i % 5 == 0 else 3 + i % 60, 1100 - i % 7]
        rows += [1, 1 + i % 2, 0]
    c = kv_case.make(form, 32, H, 64, lens, rows, seed=3)
    check(ec, c, 1, 1, 1000 if chunks else None)


@FORMS
@pytest.mark.parametrize("chunks", [False, True])
def test_tables_that_pass_31_bits(ec, form, chunks):
    """A table of 2^31 positions, one page over and over: the longest sequence is taken as far
    as 31 bits go, and the one beside it is as ever."""
    import torch
    c = kv_case.make(form, 128, 1, 64, [200, 128], [2, 1], seed=4)
    q = kv_case.queries(3, 64, 4)
    want, mass = P.attend(c.pages, c.scale, c.table, c.lens, c.row0, q, 1, 1)
    pool, batch = c.device(ec)
    table = torch.full((2, 2 ** 24), int(c.table[1, 0]), dtype=torch.int32, device="cuda")
    table[0, :2] = batch.table[0]
    for n, status in ((128, 0), (2 ** 31 - 128, 0), (2 ** 31 - 127, 8), (2 ** 31 - 1, 8)):
        lens = torch.tensor([200, n], dtype=torch.int32, device="cuda")
        wide = ec.KVBatch(table, lens, batch.row0, 3, 1000 if chunks else 2)
        out = ec.echo_kv_attention(pool, wide, torch.from_numpy(q).to("cuda", torch.bfloat16), causal_block=1)
        out = out.float().cpu().numpy()
        assert ec.echo_get_device_error() == status and np.isfinite(out).all()
        rows = 3 if n == 128 else 2
        assert (np.abs(out - want)[:rows] <= TOL * mass[:rows] + 1e-30).all()
