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


def check(ec, c, group, cb, max_rows=None, table=None):
    """Against the oracle, and the same bits again."""
    Hq = c.H * group
    q = kv_case.queries(c.n_rows, Hq * c.d, 1, 1.5)
    want, mass = P.attend(c.values, None, c.table, c.lens, c.row0, q, Hq, cb)
    pool, batch = c.device(ec, max_rows)
    if table is not None:
        batch = table(ec, c, batch, max_rows)
    out = attend(ec, pool, batch, bf(q), Hq, cb)
    assert ec.echo_get_device_error() == 0
    bad = ~(np.abs(out - want) <= TOL * mass + 1e-30)
    assert not bad.any(), (int(bad.sum()), np.argwhere(bad.any(axis=1)).ravel()[:8].tolist())
    assert np.array_equal(out, attend(ec, pool, batch, bf(q), Hq, cb))


# ---- the division of work, as test_gpu_kv_division.py has it for the other forms ----

WAYS = pytest.mark.parametrize("d,chunks,table", [(64, False, None), (64, False, wide), (64, True, None),
                                                  (128, False, None), (128, True, None)])


@WAYS
@pytest.mark.parametrize("left", [1, 8])
def test_equal_items_and_a_few_more(ec, d, chunks, table, left):
    """One item for every CTA and a few over: CTAs get one unit of those, or none."""
    items = sms() * (1 if chunks else 2) + left
    H = max(h for h in range(1, 10) if items % h == 0)
    n = 1200 if chunks else 900
    c = int4_case.make(128, H, d, [n] * (items // H), [1] * (items // H), seed=left)
    check(ec, c, 1, 1, 1000 if chunks else 1, table)


@WAYS
@pytest.mark.parametrize("seqs", [4, 50, 700])
def test_ragged_items_in_rounds(ec, d, chunks, table, seqs):
    """More than two items for every CTA, no more sequences than a block has warps, more
    than that, and more than it has threads."""
    g = np.random.default_rng(seqs)
    H = -(-int(2.3 * sms() * (1 if chunks else 2)) // seqs)
    lens = [int(n) for n in g.integers(700, 1100 if chunks else 900, seqs)]
    lens[seqs // 2] = 1100 if chunks else 900
    rows = [int(r) for r in g.integers(1, 4, seqs)]
    c = int4_case.make(16, H, d, lens, rows, seed=seqs)
    check(ec, c, 1, 1, 1000 if chunks else 3, table)


@HEADS
def test_tiles_of_long_chunks_in_rounds(ec, d):
    """Several tiles of a sequence, which see more keys from tile to tile."""
    H = -(-sms() * 13 // 50)
    c = int4_case.make(64, H, d, [1200, 1100], [600, 300], seed=2)
    check(ec, c, 1, 1, 600)


@WAYS
def test_items_without_keys_among_rounds(ec, d, chunks, table):
    """Sequences that are empty, short, or without rows between the others."""
    items = sms() * (1 if chunks else 2)
    H = 6
    lens, rows = [], []
    for i in range(items // H):
        lens += [1100 if i % 3 else 1090, 0 if i % 5 == 0 else 3 + i % 60, 1100 - i % 7]
        rows += [1, 1 + i % 2, 0]
    c = int4_case.make(32, H, d, lens, rows, seed=3)
    check(ec, c, 1, 1, 1000 if chunks else 2, table)


# ---- blocks of 256 keys ----

BORDERS = [1, 31, 32, 33, 63, 64, 65, 127, 128, 129, 191, 193, 255, 256, 257, 300, 511, 512, 513, 769, 1025, 0, 2049]


@PAGES
@pytest.mark.parametrize("group,rows,cb", [(1, 1, 1), (8, 1, 0), (3, 1, 1), (2, 4, 1), (1, 8, 1), (1, 7, 24), (2, 3, 0)])
def test_blocks_of_256_keys(ec, page, group, rows, cb):
    """Lengths around the borders of a warp's 64 keys, of a block, and of several."""
    c = int4_case.make(page, 2, 64, BORDERS, [rows] * len(BORDERS), seed=group + page)
    check(ec, c, group, cb, rows, wide)


@PAGES
@pytest.mark.parametrize("n", [20001, 20224])
def test_a_long_sequence_in_pieces(ec, page, n):
    """One sequence that many CTAs share, beside a short one."""
    c = int4_case.make(page, 1, 64, [n, 5], [2, 1], seed=page)
    check(ec, c, 4, 1, 2, wide)


def test_full_tables(ec):
    """A call that takes these blocks by its own lengths: sequences that fill their tables."""
    n = 2 * sms() * 16 * 256 // (8 * 8) + 64
    c = int4_case.make(64, 8, 64, [n - 3 * i for i in range(8)], [1] * 8, seed=5)
    check(ec, c, 1, 1, 1)


@PAGES
@pytest.mark.parametrize("kv", [0, 1])
@pytest.mark.parametrize("value", [np.inf, np.nan])
def test_scales_that_are_not_finite(ec, page, kv, value):
    """NaN in a key, or a value that is not finite, makes the rows that see it not finite (an infinite key
    may give a score of -infinity, and a weight of 0), and changes nothing in the others."""
    lens, rows = [1000, 90], [3, 4]
    base = int4_case.make(page, 2, 64, lens, rows, seed=7)
    q = kv_case.queries(base.n_rows, 2 * 64, 8, 1.5)
    want, mass = P.attend(base.values, None, base.table, base.lens, base.row0, q, 2, 1)
    for b, p in ((0, 3), (0, 255), (0, 256), (0, 998), (0, 999), (1, 88)):
        c = int4_case.make(page, 2, 64, lens, rows, seed=7)
        c.scale[c.table[b, p // page], kv, 1, p % page, 1] = value
        pool, batch = c.device(ec)
        got = attend(ec, pool, wide(ec, c, batch, 4), bf(q), 2, 1)
        assert ec.echo_get_device_error() == 0
        for r, s, pos in P.rows_of(base.lens, base.row0, base.table.shape[1], page):
            spoilt = s == b and pos >= p
            fine = slice(0, 64) if spoilt else slice(0, 128)
            if spoilt and not (kv == 0 and value == np.inf):
                assert not np.isfinite(got[r, 64:]).all()
            assert (np.abs(got[r, fine] - want[r, fine]) <= TOL * mass[r, fine] + 1e-30).all()


def test_captured_and_replayed(ec):
    """In a graph, replayed with other queries and lengths."""
    import torch
    c = int4_case.make(16, 2, 64, [700, 300], [1, 1], seed=4)
    pool, batch = c.device(ec)
    batch = wide(ec, c, batch, 1)
    q = bf(kv_case.queries(2, 128, 4))
    out = torch.empty_like(q)
    ws = torch.empty(ec.echo_kv_attention_workspace_size(pool, batch, 2), dtype=torch.uint8, device="cuda")
    step = lambda: ec.echo_kv_attention(pool, batch, q, causal_block=1, out=out, workspace=ws)   # noqa: E731
    step()
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        step()
    for i, lens in enumerate(([700, 300], [257, 1], [512, 299])):
        new = kv_case.queries(2, 128, 10 + i)
        q.copy_(bf(new))
        batch.lens.copy_(torch.tensor(lens, dtype=torch.int32))
        g.replay()
        torch.cuda.synchronize()
        want, mass = P.attend(c.values, None, c.table, np.array(lens, np.int32), c.row0, new, 2, 1)
        assert (np.abs(out.float().cpu().numpy() - want) <= TOL * mass + 1e-30).all()
    assert ec.echo_get_device_error() == 0
