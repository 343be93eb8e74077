"""Page tables and slot maps built on the GPU, number for number against the oracle's
bookkeeping; calls that cannot be served change nothing; captured steps."""
import numpy as np
import pytest

pytestmark = pytest.mark.gpu

from oracle import tables as T                     # noqa: E402


@pytest.fixture(scope="module")
def ec():
    import torch
    if not torch.cuda.is_available():
        pytest.skip("needs a GPU")
    from paper_2608_02474_gb300 import echocache
    return echocache


def i32(a):
    import torch
    return torch.tensor(list(a), dtype=torch.int32, device="cuda")


def pair(ec, n_pages, page, n_slots, max_pages, seed=None):
    """Empty tables on the GPU and the oracle's; with a seed, the stack in another order."""
    t = ec.KVTables.empty(n_pages, page, n_slots, max_pages)
    free = None
    if seed is not None:
        free = np.random.default_rng(seed).permutation(n_pages)
        t.free_pages.copy_(i32(free))
    return t, T.Tables(n_pages, page, n_slots, max_pages, free=free)


def same_tables(t, o):
    assert t.lens.tolist() == o.lens and t.n_free.tolist() == [len(o.free)]
    assert t.free_pages.tolist()[:len(o.free)] == o.free
    table = t.table.cpu().numpy()
    for s, pages in enumerate(o.pages):
        assert table[s, :len(pages)].tolist() == pages


def extend(ec, t, o, slots, rows, n_rows, seed=0):
    """One call on both; returns the step."""
    import torch
    step = ec.KVStep.empty(t, len(rows), n_rows, max(rows, default=0))
    step.batch.table.fill_(-7)
    ec.echo_kv_extend(t, i32(rows), step, None if slots is None else i32(slots))
    ids = list(range(len(rows))) if slots is None else slots
    want = o.extend(ids, rows, n_rows)
    assert want is not None
    lens, row0, maps = want
    assert step.batch.lens.tolist() == lens and step.batch.row0.tolist() == row0
    assert step.place.dtype == torch.int64
    got = torch.stack([step.place, step.pos.long(), step.seq.long()], dim=1).cpu().numpy()
    assert np.array_equal(got, np.array(maps, dtype=np.int64).reshape(-1, 3))
    table = step.batch.table.cpu().numpy()
    for b, s in enumerate(ids):
        n = len(o.pages[s])
        assert table[b, :n].tolist() == o.pages[s] and (table[b, n:] == -7).all()
    same_tables(t, o)
    return step


@pytest.mark.parametrize("page", [16, 32, 64, 128])
@pytest.mark.parametrize("rows,pad", [([1], 0), ([0], 3), ([17, 0, 1, 200], 5), ([1] * 70, 0), ([5000], 0),
                                      ([0, 0, 3, 0], 1), ([33] * 40, 100)])
def test_grow_and_shrink(ec, page, rows, pad):
    B, n = len(rows), sum(rows)
    t, o = pair(ec, 2 * (n // page + 2 * B + 2), page, B + 3, n // page + 4, seed=B)
    g = np.random.default_rng(B)
    slots = [int(s) for s in g.permutation(B + 3)[:B]]
    extend(ec, t, o, slots, rows, n + pad)
    extend(ec, t, o, slots[::-1], [min(r, 9) for r in rows], n + pad)
    for cut in ([r // 2 for r in rows], [0] * B, [2 ** 31 - 1] * B):
        ec.echo_kv_shorten(t, i32(cut), i32(slots))
        assert o.shorten(slots, cut)
        same_tables(t, o)
    assert ec.echo_get_device_error() == 0


def test_random_walk(ec):
    """Many calls in a row, some of which cannot be served."""
    g = np.random.default_rng(8)
    t, o = pair(ec, 120, 16, 12, 30)
    refused = 0
    for _ in range(150):
        B = int(g.integers(1, 13))
        slots = [int(s) for s in g.permutation(12)[:B]]
        rows = [int(r) for r in g.integers(0, 90, B)]
        if g.random() < 0.45:
            ec.echo_kv_shorten(t, i32(rows), i32(slots))
            assert o.shorten(slots, rows)
            same_tables(t, o)
            continue
        n = sum(rows) + int(g.integers(0, 4))
        keep = T.Tables(120, 16, 12, 30, free=o.free)
        keep.pages, keep.lens = [list(p) for p in o.pages], list(o.lens)
        if keep.extend(slots, rows, n) is not None:
            extend(ec, t, o, slots, rows, n)
            continue
        refused += 1
        step = ec.KVStep.empty(t, B, n)
        ec.echo_kv_extend(t, i32(rows), step, i32(slots))
        assert ec.echo_get_device_error() == 8
        same_tables(t, o)
        assert not step.batch.row0.any() and bool((step.place == -1).all()) and bool((step.pos == -1).all())
    assert refused > 5 and ec.echo_get_device_error() == 0


def test_many_sequences(ec):
    """More than one pass of the sums, and a large cluster's worth of entries."""
    g = np.random.default_rng(9)
    for B in (1024, 1025, 5000, 8192):
        rows = [int(r) for r in g.integers(0, 60, B)]
        t, o = pair(ec, sum(rows) // 16 + 2 * B, 16, B + 5, 10, seed=1)
        slots = [int(s) for s in g.permutation(B + 5)[:B]]
        extend(ec, t, o, slots, rows, sum(rows) + 1)
        extend(ec, t, o, None, [1] * B, B)
        ec.echo_kv_shorten(t, i32([41] * B), i32(slots))
        assert o.shorten(slots, [41] * B)
        same_tables(t, o)
    assert ec.echo_get_device_error() == 0


@pytest.mark.parametrize("rows,pad", [([9000], 1), ([8190, 0, 0, 1, 2], 2), ([3] * 3000, 6), ([0, 0, 20011, 0], 0)])
def test_many_rows(ec, rows, pad):
    """Row maps of a launch of their own; refused calls; maps that are not wanted, or lie anywhere."""
    import ctypes
    import torch
    B, n = len(rows), sum(rows)
    t, o = pair(ec, n // 16 + 2 * B + 5, 16, B + 2, n // 16 + 3, seed=3)
    slots = [int(s) for s in np.random.default_rng(4).permutation(B + 2)[:B]]
    extend(ec, t, o, slots, rows, n + pad)
    extend(ec, t, o, None, [min(r, 1) for r in rows], n + pad)
    step = ec.KVStep.empty(t, B, n + pad)
    ec.echo_kv_extend(t, i32([n + pad + 1] + [0] * (B - 1)), step, i32(slots))
    assert ec.echo_get_device_error() == 8 and bool((step.place == -1).all()) and bool((step.seq == -1).all())
    same_tables(t, o)
    # four bytes further on, and without places and sequences
    wide = torch.full((n + pad + 9,), -9, dtype=torch.int32, device="cuda")
    few = [min(r, 2) for r in rows]
    lens, row0 = i32([0] * B), i32([0] * (B + 1))
    assert ec.lib().echo_kv_extend(ctypes.byref(t.cstruct), i32(slots).data_ptr(), i32(few).data_ptr(), B, n + pad, None,
                                   lens.data_ptr(), row0.data_ptr(), None, wide.data_ptr() + 4, None,
                                   torch.cuda.current_stream().cuda_stream) == 0
    _, _, maps = o.extend(slots, few, n + pad)
    assert wide.tolist() == [-9] + [m[1] for m in maps] + [-9] * 8
    same_tables(t, o)


def test_tokens_past_31_bits_in_all(ec):
    """Shortening sequences whose lengths sum to more than 2^31 (their tables are only read
    where pages are given back)."""
    import torch
    n, page, width = 9, 128, 2 ** 21
    t = ec.KVTables(torch.zeros(n, width, dtype=torch.int32, device="cuda"), i32([width * page - 128] * n),
                    torch.zeros(100, dtype=torch.int32, device="cuda"), i32([0]), page)
    t.table[:, width - 2] = torch.arange(n, device="cuda", dtype=torch.int32) + 50
    ec.echo_kv_shorten(t, i32([5] * n))
    assert t.lens.tolist() == [width * page - 133] * n and t.n_free.tolist() == [0]
    ec.echo_kv_shorten(t, i32([123] * n))
    assert t.n_free.tolist() == [n] and t.free_pages.tolist()[:n] == [58, 57, 56, 55, 54, 53, 52, 51, 50]
    assert t.lens.tolist() == [width * page - 256] * n and ec.echo_get_device_error() == 0
    ec.echo_kv_shorten(t, i32([2 ** 31 - 1] * n))       # more pages than the pool has: no tables of it
    assert ec.echo_get_device_error() == 8 and t.n_free.tolist() == [n]
    assert t.lens.tolist() == [width * page - 256] * n


@pytest.mark.parametrize("slots,rows,n_rows", [
    ([1, 1], [1, 1], 2), ([0, 4], [1, 1], 2), ([0, -1], [1, 1], 2), ([0, 1], [1, -1], 2), ([0, 1], [2, 1], 2),
    ([0, 1], [200, 1], 300), ([0, 1], [100, 100], 300), ([2 ** 31 - 1, 1], [1, 1], 2),
    ([0, 1], [2 ** 31 - 1, 2 ** 31 - 1], 2)])
def test_calls_that_cannot_be_served(ec, slots, rows, n_rows):
    t, o = pair(ec, 10, 16, 4, 9)
    extend(ec, t, o, [2, 1], [20, 5], 25)
    step = ec.KVStep.empty(t, 2, n_rows)
    step.batch.table.fill_(-7)
    ec.echo_kv_extend(t, i32(rows), step, i32(slots))
    assert ec.echo_get_device_error() == 8
    same_tables(t, o)
    assert step.batch.row0.tolist() == [0, 0, 0] and bool((step.batch.table == -7).all())
    for m in (step.place, step.pos, step.seq):
        assert bool((m == -1).all())
    if len(set(slots)) < 2 or min(rows) < 0 or not set(slots) <= {0, 1, 2, 3}:
        ec.echo_kv_shorten(t, i32(rows), i32(slots))
        assert ec.echo_get_device_error() == 8
        same_tables(t, o)


def test_tables_that_are_none(ec):
    for n_free, lens in ((-1, [0, 0]), (11, [0, 0]), (5, [-1, 0]), (5, [2 ** 30, 0])):
        t = ec.KVTables.empty(10, 16, 2, 4)
        t.n_free.fill_(n_free)
        t.lens.copy_(i32(lens))
        step = ec.KVStep.empty(t, 2, 4)
        ec.echo_kv_extend(t, i32([1, 1]), step)
        assert ec.echo_get_device_error() == 8 and t.lens.tolist() == lens and t.n_free.tolist() == [n_free]
        ec.echo_kv_shorten(t, i32([1, 1]))
        assert ec.echo_get_device_error() == 8 and t.lens.tolist() == lens and t.n_free.tolist() == [n_free]


def test_no_sequences(ec):
    t, o = pair(ec, 4, 16, 2, 2)
    extend(ec, t, o, [], [], 3)
    ec.echo_kv_shorten(t, i32([]))
    same_tables(t, o)
    assert ec.echo_get_device_error() == 0


def test_a_captured_step(ec):
    """One graph that takes a token a sequence, replayed over page borders, and its rows in the pool's
    tables; the next capture shares the tables."""
    import torch
    t, o = pair(ec, 40, 16, 3, 12)
    extend(ec, t, o, [0, 1, 2], [15, 30, 0], 45)
    rows, step = i32([1, 2, 1]), ec.KVStep.empty(t, 3, 4, 2)
    ec.echo_kv_extend(t, rows, step)                     # a first call outside
    o.extend([0, 1, 2], [1, 2, 1], 4)
    torch.cuda.synchronize()
    g, back = torch.cuda.CUDAGraph(), torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        ec.echo_kv_extend(t, rows, step)
    with torch.cuda.graph(back):
        ec.echo_kv_shorten(t, rows)
    for i in range(40):
        (back if i % 5 == 4 else g).replay()
        if i % 5 == 4:
            o.shorten([0, 1, 2], [1, 2, 1])
        else:
            _, _, maps = o.extend([0, 1, 2], [1, 2, 1], 4)
            assert step.place.tolist() == [m[0] for m in maps] and step.pos.tolist() == [m[1] for m in maps]
        same_tables(t, o)
    assert ec.echo_get_device_error() == 0


def test_another_stream(ec):
    import torch
    s = torch.cuda.Stream()
    with torch.cuda.stream(s):
        rows = i32([3, 40])
    t = ec.KVTables.empty(10, 16, 2, 5, stream=s)
    step = ec.KVStep.empty(t, 2, 43, stream=s)
    ec.echo_kv_extend(t, rows, step, stream=s)
    ec.echo_kv_shorten(t, rows, stream=s)
    s.synchronize()
    assert step.batch.lens.tolist() == [3, 40] and t.lens.tolist() == [0, 0] and t.n_free.tolist() == [10]
