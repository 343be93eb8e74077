"""Attention over the paged key/value cache against the oracle in fp64.

Tolerance.  Every weight p is rounded to bf16 (for int8 pages times its value's scale)
before the product with v, and the result is rounded to bf16: bf16 numbers have 8
significant bits, so each is off by up to 2^-8, of mass = sum_j p_j |v_j| and of
|out| <= mass.  The fp32 parts (scores, exponentials, sums, the rescaling between key
ranges) stay below 0.15 * 2^-8 at these sizes: a score's absolute error is at most a few
2^-24 of its size times the terms of its sum, here below 1e-4 in the exponent even for
scores of a few hundred.  So element by element |out - oracle| <= 2.15 * 2^-8 * mass.
"""
import numpy as np
import pytest

pytestmark = pytest.mark.gpu

import kv_case                                     # noqa: E402
from oracle import paged as P                      # noqa: E402

F32 = np.float32
TOL = 2.15 * 2.0 ** -8


@pytest.fixture(scope="module")
def ec():
    import torch
    if not torch.cuda.is_available():
        pytest.skip("needs a GPU")
    from paper_2608_02474_gb300 import echocache
    return echocache


def bf(a):
    import torch
    return torch.from_numpy(np.ascontiguousarray(a)).to("cuda", torch.bfloat16)


def close(got, want, mass):
    assert np.isfinite(got).all()
    bad = np.abs(got - want) > TOL * mass + 1e-30
    assert not bad.any(), (int(bad.sum()), np.argwhere(bad)[:5].tolist(),
                           float((np.abs(got - want) / np.maximum(mass, 1e-30)).max()))


def run(ec, c, q, Hq, cb, max_rows=None):
    pool, batch = c.device(ec, max_rows)
    out = ec.echo_kv_attention(pool, batch, bf(q), causal_block=cb)
    again = ec.echo_kv_attention(pool, batch, bf(q), causal_block=cb)
    assert ec.echo_get_device_error() == 0
    assert (out == again).all()                      # the same bits every time
    return out.float().cpu().numpy()


def check(ec, c, group, cb, seed=0, scale=1.5, max_rows=None):
    Hq = c.H * group
    q = kv_case.queries(c.n_rows, Hq * c.d, seed, scale)
    want, mass = P.attend(c.pages, c.scale, c.table, c.lens, c.row0, q, Hq, cb)
    close(run(ec, c, q, Hq, cb, max_rows), want, mass)


FORMS = pytest.mark.parametrize("form", ["bf16", "int8"])
HEADS = pytest.mark.parametrize("d", [64, 128])


@FORMS
@HEADS
@pytest.mark.parametrize("page", [16, 32, 64, 128])
@pytest.mark.parametrize("n", [1, 15, 16, 17, 63, 64, 65, 127, 128, 129, 500])
def test_single_tokens(ec, form, d, page, n):
    """One new token of two sequences, lengths around pages and key blocks."""
    check(ec, kv_case.make(form, page, 2, d, [n, n + 1], [1, 1], seed=n), 2, 1)


@FORMS
@HEADS
@pytest.mark.parametrize("group", [1, 2, 3, 5, 7, 8, 16, 17, 33])
def test_shared_heads(ec, form, d, group):
    check(ec, kv_case.make(form, 32, 2, d, [300, 77], [1, 2], seed=group), group, 1)


@FORMS
@HEADS
@pytest.mark.parametrize("lens,rows,cb", [
    ([200], [200], 1),                  # a prompt of its own
    ([700], [130], 1),                  # a chunk, two tiles, the second of two rows
    ([700], [130], 0),
    ([513], [257], 100),                # causal by frames that the chunk cuts
    ([129], [128], 128),
    ([40, 0, 300, 7], [17, 0, 40, 7], 1),
    ([40, 300, 0, 7], [40, 1, 0, 3], 0),
    ([30], [50], 1),                    # rows before the start of the sequence
    ([20], [300], 0),                   # more queries than keys: cross-attention
    ([0, 5], [40, 40], 0),              # no key at all
    ([0, 5], [40, 40], 1),
    ([1500, 2, 900], [1, 1, 33], 1),
])
@pytest.mark.parametrize("group", [1, 4])
def test_chunks(ec, form, d, lens, rows, cb, group):
    c = kv_case.make(form, 16 if d == 64 else 64, 2, d, lens, rows, seed=len(lens) + rows[0])
    check(ec, c, group, cb)


@FORMS
@HEADS
@pytest.mark.parametrize("rows", [1, 20])
@pytest.mark.parametrize("max_rows", [0, 1, 8, 100000])
def test_any_max_rows_is_right(ec, form, d, rows, max_rows):
    check(ec, kv_case.make(form, 32, 1, d, [150, 90], [rows, 3 * rows], seed=9), 2, 1,
          max_rows=max_rows)


@FORMS
@HEADS
@pytest.mark.parametrize("rows", [1, 64])
def test_long_axis(ec, form, d, rows):
    """Few rows, many keys: the keys are split over the SMs and joined."""
    check(ec, kv_case.make(form, 128, 1, d, [9001, 1, 4097], [rows, 1, 1], seed=3), 3, 1)


@FORMS
@HEADS
def test_many_sequences(ec, form, d):
    """More sequences than one search step holds, some without rows or keys."""
    g = np.random.default_rng(5)
    lens = [int(n) for n in g.integers(0, 90, 300)]
    rows = [int(r) for r in g.integers(0, 3, 300)]
    check(ec, kv_case.make(form, 16, 1, d, lens, rows, seed=6), 2, 1)


@FORMS
@HEADS
@pytest.mark.parametrize("rows", [1, 150])
def test_late_maxima(ec, form, d, rows):
    """Keys late in the sequence whose scores exceed the first ones by far more than 2^64
    in the exponential, for some rows only: every running maximum has to move."""
    c = kv_case.make(form, 32, 1, d, [700], [rows], seed=11, amplitude=0.1)
    q = kv_case.queries(rows, 2 * d, 12, 0.3) + F32(2.0)
    q[::2] *= -1
    q = kv_case.G.to_bf16_values(q)
    for p, a in ((300, 3.0), (301, -3.0), (555, 6.0), (600, -7.0)):
        pg, at = c.table[0, p // 32], p % 32
        if form == "int8":
            c.pages[pg, 0, 0, at] = 127 if a > 0 else -127
            c.scale[pg, 0, 0, at] = abs(a) / 127
        else:
            c.pages[pg, 0, 0, at] = a
    want, mass = P.attend(c.pages, c.scale, c.table, c.lens, c.row0, q, 2, 0)
    close(run(ec, c, q, 2, 0), want, mass)


@FORMS
@HEADS
@pytest.mark.parametrize("lens,rows", [([1300], [150]), ([129, 128, 300], [128, 200, 129])])
def test_maxima_in_every_block(ec, form, d, lens, rows):
    """One key of every 64, and the last, whose score exceeds the earlier ones by far more
    than 2^64, up for even rows and down for odd ones: the maximum moves in every block of
    every tile, the last one too."""
    c = kv_case.make(form, 64, 1, d, lens, rows, seed=13, amplitude=0.1)
    q = kv_case.queries(sum(rows), 2 * d, 14, 0.3) + F32(2.0)
    q[::2] *= -1
    q = kv_case.G.to_bf16_values(q)
    for b, n in enumerate(lens):
        for i, p in enumerate([*range(37, n, 64), n - 1]):
            a, pg = (1.0 + 3 * i) * (-1) ** i, c.table[b, p // 64]
            if form == "int8":
                c.pages[pg, 0, 0, p % 64] = 127 if a > 0 else -127
                c.scale[pg, 0, 0, p % 64] = abs(a) / 127
            else:
                c.pages[pg, 0, 0, p % 64] = a
    want, mass = P.attend(c.pages, c.scale, c.table, c.lens, c.row0, q, 2, 0)
    close(run(ec, c, q, 2, 0, max_rows=1000), want, mass)


@FORMS
@HEADS
@pytest.mark.parametrize("cb", [0, 1])
def test_many_short_items_of_the_chunk_kernel(ec, form, d, cb):
    """More items of one to four key blocks than CTAs, by the kernel for many rows."""
    g = np.random.default_rng(15)
    lens = [int(n) for n in g.integers(1, 450, 260)]
    rows = [int(r) for r in g.integers(0, 4, 260)]
    check(ec, kv_case.make(form, 16, 3, d, lens, rows, seed=16), 2, cb, max_rows=1000)


@FORMS
@HEADS
@pytest.mark.parametrize("rows", [1, 40])
def test_strided_rows_and_columns_beyond(ec, form, d, rows):
    """q as columns of a wider tensor, out into one: nothing beyond its columns changes."""
    import torch
    c = kv_case.make(form, 16, 2, d, [100, 60], [rows, rows], seed=13)
    q = kv_case.queries(c.n_rows, 4 * d, 13)
    want, mass = P.attend(c.pages, c.scale, c.table, c.lens, c.row0, q, 4, 1)
    pool, batch = c.device(ec)
    wide = torch.full((c.n_rows, 8 * d + 8), float("nan"), dtype=torch.bfloat16, device="cuda")
    wide[:, 8:8 + 4 * d] = bf(q)
    dst = torch.full((c.n_rows + 1, 4 * d + 16), 5.0, dtype=torch.bfloat16, device="cuda")
    ec.echo_kv_attention(pool, batch, wide[:, 8:8 + 4 * d], causal_block=1, out=dst[:-1, 8:8 + 4 * d])
    close(dst[:-1, 8:8 + 4 * d].float().cpu().numpy(), want, mass)
    assert bool((dst[:, :8] == 5).all()) and bool((dst[:, 8 + 4 * d:] == 5).all())
    assert bool((dst[-1] == 5).all()) and ec.echo_get_device_error() == 0


@FORMS
@HEADS
def test_rows_of_no_sequence_are_left_alone(ec, form, d):
    import torch
    c = kv_case.make(form, 16, 1, d, [50], [30], seed=14)
    pool, batch = c.device(ec)
    for max_rows in (1, 30):
        batch = ec.KVBatch(batch.table, batch.lens, batch.row0, 45, max_rows)
        q = kv_case.queries(45, d, 14)
        out = torch.full((45, d), 7.0, dtype=torch.bfloat16, device="cuda")
        ec.echo_kv_attention(pool, batch, bf(q), out=out, causal_block=1)
        want, mass = P.attend(c.pages, c.scale, c.table, c.lens, c.row0, q[:30], 1, 1)
        close(out[:30].float().cpu().numpy(), want, mass)
        assert bool((out[30:] == 7).all())
    assert ec.echo_get_device_error() == 0


@FORMS
@HEADS
@pytest.mark.parametrize("rows", [1, 40])
def test_page_outside_the_pool(ec, form, d, rows):
    """The flag, and the other sequence's rows as ever."""
    c = kv_case.make(form, 16, 1, d, [100, 100], [rows, rows], seed=15)
    c.pages = np.nan_to_num(c.pages) if form == "bf16" else c.pages
    c.scale = np.nan_to_num(c.scale) if form == "int8" else None
    q = kv_case.queries(2 * rows, d, 15)
    want, mass = P.attend(c.pages, c.scale, c.table, c.lens, c.row0, q, 1, 1)
    for page in (-1, c.pages.shape[0], 2 ** 31 - 1, -2 ** 31):
        pool, batch = c.device(ec)
        batch.table[0, 2] = page
        out = ec.echo_kv_attention(pool, batch, bf(q), causal_block=1).float().cpu().numpy()
        assert ec.echo_get_device_error() == 8
        close(out[rows:], want[rows:], mass[rows:])
    pool, batch = c.device(ec)
    batch.lens[0] = 2 ** 31 - 1                       # a length far past the table
    out = ec.echo_kv_attention(pool, batch, bf(q), causal_block=1).float().cpu().numpy()
    assert ec.echo_get_device_error() == 8
    close(out[rows:], want[rows:], mass[rows:])


@FORMS
def test_scores_of_zero_and_equal_keys(ec, form):
    """A query of zeros averages the values."""
    c = kv_case.make(form, 16, 1, 64, [333], [2], seed=16)
    q = np.zeros((2, 64), F32)
    want, mass = P.attend(c.pages, c.scale, c.table, c.lens, c.row0, q, 1, 0)
    close(run(ec, c, q, 1, 0), want, mass)


@pytest.mark.parametrize("d", [64, 128])
def test_pool_beyond_32_bits(ec, d):
    """Pages whose first byte lies past 4 GB, and whose value index lies past 2^32."""
    import torch
    page, H = 128, 8
    per = 2 * H * page * d                            # values of a page
    n_pages = (2 ** 32 + 2 ** 30) // per + 2
    pages = torch.empty(n_pages, 2, H, page, d, dtype=torch.bfloat16, device="cuda")
    c = kv_case.make("bf16", page, H, d, [200], [3], seed=17)
    c.pages = np.nan_to_num(c.pages)
    far = [n_pages - 1, 2 ** 32 // per + 1]
    for i, pg in enumerate(c.table[0]):
        pages[far[i]] = bf(c.pages[pg])
    pool = ec.KVPool(pages)
    t = lambda a: torch.tensor(a, dtype=torch.int32, device="cuda")     # noqa: E731
    for rows, k in ((3, 1), (40, 1)):
        batch = ec.KVBatch(t([far]), t([200]), t([0, rows]), rows, rows)
        q = kv_case.queries(rows, H * d, 18)
        want, mass = P.attend(c.pages, None, c.table, c.lens, [0, rows], q, H, 1)
        close(ec.echo_kv_attention(pool, batch, bf(q), causal_block=1).float().cpu().numpy(), want, mass)
    kk, _ = ec.echo_kv_read(pool, batch)
    assert torch.equal(kk[-1].view(H, d), pages[far[1], 0, :, 71])
    assert ec.echo_get_device_error() == 0


def test_other_stream_graph_and_profile(ec):
    """On a stream of its own, and captured in a graph that is replayed on new queries."""
    import torch
    c = kv_case.make("int8", 64, 4, 128, [600, 100], [2, 1], seed=19)
    pool, batch = c.device(ec)
    q = bf(kv_case.queries(3, 4 * 128, 19))
    want = ec.echo_kv_attention(pool, batch, q, causal_block=1)
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    got = ec.echo_kv_attention(pool, batch, q, causal_block=1, stream=s)
    s.synchronize()
    assert torch.equal(got, want)
    ws = torch.empty(ec.echo_kv_attention_workspace_size(pool, batch, 4), dtype=torch.uint8,
                     device="cuda")
    out = torch.empty_like(q)
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        ec.echo_kv_attention(pool, batch, q, causal_block=1, out=out, workspace=ws)
    for seed in (20, 21):
        q.copy_(bf(kv_case.queries(3, 512, seed)))
        g.replay()
        assert torch.equal(out, ec.echo_kv_attention(pool, batch, q, causal_block=1))
    assert ec.echo_get_device_error() == 0


@FORMS
@HEADS
@pytest.mark.parametrize("rows,cb", [(3, 1), (8, 4), (40, 1), (200, 1), (200, 64)])
@pytest.mark.parametrize("what", [0, 1])             # a key, a value
@pytest.mark.parametrize("value", [np.inf, np.nan])
def test_not_finite_where_only_later_rows_see_it(ec, form, d, rows, cb, what, value):
    """Rows that do not see the key are as ever; those that do are not finite (an infinite
    key may give a score of -infinity, and a weight of 0)."""
    n, at = 300, 300 - rows // 2
    c = kv_case.make(form, 16, 2, d, [n], [rows], seed=21)
    q = kv_case.queries(rows, 4 * d, 21)
    want, mass = P.attend(c.pages, c.scale, c.table, c.lens, c.row0, q, 4, cb)
    pg, slot = c.table[0, at // 16], at % 16
    if form == "int8":
        c.scale[pg, what, 1, slot] = value
    else:
        c.pages[pg, what, 1, slot, 5] = value
    pool, batch = c.device(ec)
    got = ec.echo_kv_attention(pool, batch, bf(q), causal_block=cb).float().cpu().numpy()
    sees = np.array([P.top_of(n - rows + i, n, cb) > at for i in range(rows)])
    assert sees.any() and not sees.all()
    close(got[:, :2 * d], want[:, :2 * d], mass[:, :2 * d])      # the other key/value head
    close(got[~sees], want[~sees], mass[~sees])
    if what == 1 or np.isnan(value):
        assert not np.isfinite(got[sees][:, [2 * d + 5, 3 * d + 5]]).any()
    assert ec.echo_get_device_error() == 0


@FORMS
@HEADS
@pytest.mark.parametrize("group", [1, 40])
def test_many_items_without_keys(ec, form, d, group):
    """More of them in a row than a CTA hands out at once, before, between and after others."""
    lens = [0] * 30 + [200] + [0] * 25 + [3, 400] + [0] * 17
    rows = [3] * len(lens)
    check(ec, kv_case.make(form, 16, 2, d, lens, rows, seed=23), group, 0)
    check(ec, kv_case.make(form, 16, 2, d, lens, rows, seed=24), group, 2)
