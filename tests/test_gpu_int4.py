"""The 4-bit key/value cache on the GPU: codes, scales and values bit for bit against the
oracle, and attention over them.

Tolerance of the attention.  Codes times scales are exact in bf16, so that what is said in
test_gpu_kv_attention of bf16 pages holds here: a weight p and the result are rounded to
bf16 once each, by up to 2^-8 of p and of |out| <= mass = sum_j p_j |v_j|, and the fp32
parts stay below 0.15 * 2^-8 of mass: |out - oracle| <= 2.15 * 2^-8 * mass.
"""
import numpy as np
import pytest

pytestmark = pytest.mark.gpu

import int4_case                                   # noqa: E402
import kv_case                                     # noqa: E402
from oracle import cache as C                      # noqa: E402
from oracle import int4 as I                       # noqa: E402
from oracle import paged as P                      # noqa: E402

F32 = np.float32
TOL = 2.15 * 2.0 ** -8
HEADS = pytest.mark.parametrize("d", [64, 128])


@pytest.fixture(scope="module")
def ec():
    import torch
    if not torch.cuda.is_available():
        pytest.skip("needs a GPU")
    from paper_2608_02474_gb300 import echocache
    return echocache


def host(t):
    return t.float().cpu().numpy() if t.is_floating_point() else t.cpu().numpy()


def same(a, b):
    return np.array_equal(a, b, equal_nan=a.dtype.kind == "f")


def bf(a):
    import torch
    return torch.from_numpy(np.ascontiguousarray(a)).to("cuda", torch.bfloat16)


def sources(n, cols, dtype, seed, most=1.0):
    """k and v as the two halves of one wider tensor, and their host values."""
    import torch
    x = np.random.default_rng(seed).standard_normal((n, 2 * cols)).astype(F32) * F32(most)
    x[:, ::7] *= 8
    x[:, 5::9] = np.round(x[:, 5::9] * 4) / 4       # halves between codes
    if n > 1:
        x[1, :cols // 2] = 0
    t = torch.from_numpy(x).cuda().to(torch.bfloat16 if dtype == "bf16" else torch.float32)
    return t[:, :cols], t[:, cols:], host(t[:, :cols]), host(t[:, cols:])


def written(c, k, v, rows=None):
    """The case's pages and scales with the rows written, by the oracle."""
    pages, scale = c.pages.copy(), c.scale.copy()
    for r, b, p in P.rows_of(c.lens, c.row0, c.table.shape[1], c.page):
        if rows is not None and r not in rows:
            continue
        pg, at = int(c.table[b, p // c.page]), p % c.page
        for i, src in enumerate((k, v)):
            q, s, _ = I.quantize(src[r, :c.H * c.d].reshape(c.H, c.d))
            pages[pg, i, :, at], scale[pg, i, :, at] = I.pack(q), s
    return pages, scale


CASES = [
    # page, H, d, lens, rows
    (16, 1, 64, [1], [1]),
    (64, 40, 128, [200], [9]),
    (128, 5, 128, [129, 0, 128, 300], [129, 0, 1, 77]),
    (32, 16, 64, [33, 31, 200], [2, 31, 100]),
    (16, 3, 128, list(range(1, 40)), [1] * 39),
]


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("page,H,d,lens,rows", CASES)
def test_write_and_read(ec, page, H, d, lens, rows, dtype):
    import torch
    c = int4_case.make(page, H, d, lens, rows)
    pool, batch = c.device(ec)
    k, v, hk, hv = sources(c.n_rows, H * d, dtype, seed=page + H)
    ec.echo_kv_write(pool, batch, k, v)
    pages, scale = written(c, hk, hv)
    assert same(host(pool.pages), pages) and same(host(pool.scale), scale)
    want = P.read(I.values(pages, scale), None, c.table, c.lens, c.row0, c.n_rows)
    for t in (torch.bfloat16, torch.float32):
        wide = torch.full((c.n_rows, 2 * H * d + 8), 3.0, dtype=t, device="cuda")
        ec.echo_kv_read(pool, batch, k=wide[:, :H * d], v=wide[:, H * d:2 * H * d])
        assert same(host(wide[:, :2 * H * d]), np.concatenate(want, axis=1))
        assert bool((wide[:, 2 * H * d:] == 3.0).all())
    assert ec.echo_get_device_error() == 0


@pytest.mark.parametrize("most", [2.0 ** -130, 2.0 ** -115, 1e-30, 3e35])
def test_small_and_large_values(ec, most):
    """Scales at their least value (codes of what is below it are 0), and near the largest number."""
    c = int4_case.make(16, 2, 64, [9], [9])
    pool, batch = c.device(ec)
    k, v, hk, hv = sources(9, 128, "bf16", seed=5, most=most)
    ec.echo_kv_write(pool, batch, k, v)
    pages, scale = written(c, hk, hv)
    assert same(host(pool.pages), pages) and same(host(pool.scale), scale)
    assert ec.echo_get_device_error() == 0


@pytest.mark.parametrize("value", [np.inf, -np.inf, np.nan])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_non_finite_groups(ec, value, dtype):
    """Codes 0 and the |maximum| as the group's scale, the device flag; other groups unharmed."""
    c = int4_case.make(16, 3, 64, [20], [4])
    pool, batch = c.device(ec)
    k, v, hk, hv = sources(4, 192, dtype, seed=5)
    k[2, 64 + 39], hk[2, 64 + 39] = float(value), value
    ec.echo_kv_write(pool, batch, k, v)
    pages, scale = written(c, hk, hv)
    assert same(host(pool.pages), pages) and same(host(pool.scale), scale)
    assert ec.echo_get_device_error() == 5


@pytest.mark.parametrize("form", ["int4", "int8", "bf16"])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_write_at(ec, form, dtype):
    """By a slot map: the same bits as by the batch, in any order, rows of negative places
    left out, and one past the pool refused by the flag."""
    import torch
    make = (lambda: int4_case.make(32, 3, 128, [70, 33, 5], [70, 2, 5])) if form == "int4" else \
        (lambda: kv_case.make(form, 32, 3, 128, [70, 33, 5], [70, 2, 5]))
    c = make()
    pool, batch = c.device(ec)
    other, _ = make().device(ec)
    k, v, hk, hv = sources(c.n_rows, 384, dtype, seed=3)
    ec.echo_kv_write(pool, batch, k, v)
    place = torch.full((c.n_rows,), -1, dtype=torch.int64)
    for r, b, p in P.rows_of(c.lens, c.row0, c.table.shape[1], c.page):
        place[r] = int(c.table[b, p // 32]) * 32 + p % 32
    order = torch.randperm(c.n_rows, generator=torch.Generator().manual_seed(1))
    wide = torch.cat([k, v], dim=1)[order.cuda()]
    ec.echo_kv_write_at(other, place[order].cuda(), wide[:, :384], wide[:, 384:])
    assert same(host(other.pages), host(pool.pages))
    if form != "bf16":
        assert same(host(other.scale), host(pool.scale))
    # half of the rows left out, others past the pool
    c = make()
    pool, batch = c.device(ec)
    before = host(pool.pages).copy()
    ec.echo_kv_write_at(pool, torch.full((c.n_rows,), -1, dtype=torch.int64, device="cuda"), k, v)
    assert ec.echo_get_device_error() == 0 and same(host(pool.pages), before)
    for bad in (pool.n_pages * 32, 2 ** 62, -2 ** 62):
        ec.echo_kv_write_at(pool, torch.full((c.n_rows,), bad, dtype=torch.int64, device="cuda"), k, v)
        assert ec.echo_get_device_error() == (8 if bad > 0 else 0) and same(host(pool.pages), before)
    n = ec.echo_launch_count()
    ec.echo_kv_write_at(pool, place[:0].cuda(), k[:0], v[:0])
    assert ec.echo_launch_count() == n


def close(got, want, mass):
    assert np.isfinite(got).all()
    bad = np.abs(got - want) > TOL * mass + 1e-30
    assert not bad.any(), (int(bad.sum()), np.argwhere(bad)[:5].tolist(),
                           float((np.abs(got - want) / np.maximum(mass, 1e-30)).max()))


def check(ec, c, group, cb, seed=0, scale=1.5, max_rows=None):
    Hq = c.H * group
    q = kv_case.queries(c.n_rows, Hq * c.d, seed, scale)
    want, mass = P.attend(c.values, None, c.table, c.lens, c.row0, q, Hq, cb)
    pool, batch = c.device(ec, max_rows)
    out = ec.echo_kv_attention(pool, batch, bf(q), causal_block=cb)
    again = ec.echo_kv_attention(pool, batch, bf(q), causal_block=cb)
    assert ec.echo_get_device_error() == 0
    assert (out == again).all()                      # the same bits every time
    close(host(out), want, mass)


@HEADS
@pytest.mark.parametrize("page", [16, 32, 64, 128])
@pytest.mark.parametrize("n", [1, 15, 17, 31, 32, 33, 64, 65, 127, 128, 129, 500])
def test_single_tokens(ec, d, page, n):
    check(ec, int4_case.make(page, 2, d, [n, n + 1], [1, 1], seed=n), 2, 1)


@HEADS
@pytest.mark.parametrize("group", [1, 2, 3, 5, 8, 9, 16, 17, 25, 33])
def test_shared_heads(ec, d, group):
    check(ec, int4_case.make(32, 2, d, [300, 77], [1, 2], seed=group), group, 1)


@HEADS
@pytest.mark.parametrize("page", [16, 32, 64, 128])
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
    ([1500, 2, 900], [1, 1, 33], 1),
])
def test_chunks(ec, d, page, lens, rows, cb):
    check(ec, int4_case.make(page, 2, d, lens, rows, seed=len(lens) + rows[0]), 1 if page < 64 else 4, cb)


@HEADS
@pytest.mark.parametrize("rows", [1, 20])
@pytest.mark.parametrize("max_rows", [0, 1, 12, 100000])
def test_any_max_rows_is_right(ec, d, rows, max_rows):
    check(ec, int4_case.make(32, 1, d, [150, 90], [rows, 3 * rows], seed=9), 2, 1, max_rows=max_rows)


@HEADS
@pytest.mark.parametrize("rows", [1, 64])
def test_long_axis(ec, d, rows):
    check(ec, int4_case.make(128, 1, d, [9001, 1, 4097], [rows, 1, 1], seed=3), 3, 1)


@HEADS
def test_many_sequences(ec, d):
    g = np.random.default_rng(5)
    check(ec, int4_case.make(16, 1, d, [int(n) for n in g.integers(0, 90, 300)],
                             [int(r) for r in g.integers(0, 3, 300)], seed=6), 2, 1)


@HEADS
@pytest.mark.parametrize("rows", [1, 150])
def test_late_maxima(ec, d, rows):
    """Keys late in the sequence whose scores exceed the first ones by far more than 2^64 in
    the exponential, for some rows only."""
    c = int4_case.make(32, 1, d, [700], [rows], seed=11, amplitude=2.0 ** -3)
    q = kv_case.queries(rows, 2 * d, 12, 0.3) + F32(2.0)
    q[::2] *= -1
    q = kv_case.G.to_bf16_values(q)
    for p, a in ((300, 3.0), (301, -3.0), (555, 6.0), (600, -7.0)):
        pg, at = c.table[0, p // 32], p % 32
        codes, scale, _ = I.quantize(np.full((1, d), a, F32))
        c.pages[pg, 0, :, at], c.scale[pg, 0, :, at] = I.pack(codes), scale
    want, mass = P.attend(c.values, None, c.table, c.lens, c.row0, q, 2, 0)
    pool, batch = c.device(ec)
    close(host(ec.echo_kv_attention(pool, batch, bf(q))), want, mass)
    assert ec.echo_get_device_error() == 0


@HEADS
@pytest.mark.parametrize("amplitude", [2.0 ** -100, 2.0 ** 50])
def test_scales_far_from_one(ec, d, amplitude):
    """Values at the ends of what is said to work; keys of ordinary size."""
    c = int4_case.make(16, 1, d, [200], [3], seed=4)
    c.scale[:, 1] *= F32(amplitude)
    for rows in (3, 40):
        c.row0 = np.array([0, rows], np.int32)
        check(ec, c, 2, 1)


def batch_of_all(ec, batch, n):
    """The one sequence of the batch, all of its n tokens as rows."""
    import torch
    return ec.KVBatch(batch.table, batch.lens, torch.tensor([0, n], dtype=torch.int32, device="cuda"), n)


@HEADS
@pytest.mark.parametrize("rows", [1, 60])
@pytest.mark.parametrize("kv", [0, 1])
@pytest.mark.parametrize("value", [np.inf, np.nan])
def test_scales_that_are_not_finite(ec, d, rows, kv, value):
    """A spoilt key or value makes the rows that see it not finite, and changes nothing in
    the others, in blocks that all rows see whole and in those that they do not."""
    lens, at = [500, 90], [(0, 3), (0, 497), (1, 60)]
    base = int4_case.make(32, 2, d, lens, [rows, 20], seed=7)
    q = kv_case.queries(base.n_rows, 2 * d, 8, 1.5)
    for b, p in at:
        c = int4_case.make(32, 2, d, lens, [rows, 20], seed=7)
        c.scale[c.table[b, p // 32], kv, 1, p % 32, d // 32 - 1] = value
        pool, batch = c.device(ec)
        got = host(ec.echo_kv_attention(pool, batch, bf(q), causal_block=1))
        want, mass = P.attend(base.values, None, base.table, base.lens, base.row0, q, 2, 1)
        for r, s, pos in P.rows_of(base.lens, base.row0, base.table.shape[1], 32):
            if s == b and pos >= p:
                assert not np.isfinite(got[r, d:]).all()
                close(got[r, :d], want[r, :d], mass[r, :d])
            else:
                close(got[r], want[r], mass[r])
        assert ec.echo_get_device_error() == 0


@HEADS
@pytest.mark.parametrize("rows", [1, 60])
@pytest.mark.parametrize("kv", [0, 1])
@pytest.mark.parametrize("value", [np.inf, -np.inf, np.nan])
def test_values_that_are_not_finite(ec, d, rows, kv, value):
    """As echo_kv_write leaves them (codes 0 under a scale that is not finite): the rows that see the
    key are not finite in the group's columns of this head.  The other head keeps its bits.  Rows that do
    not see the key may be rounded about another maximum, since a weight that is not finite moves those of all
    of a tile's rows: both results are within TOL * mass of the exact one, and so within 2 TOL * mass of each other."""
    n = 300
    base = int4_case.make(32, 2, d, [n], [rows], seed=9)
    q = bf(kv_case.queries(rows, 2 * d, 10, 1.5))
    pool, batch = base.device(ec)
    every = batch_of_all(ec, batch, n)
    kept = ec.echo_kv_read(pool, every)
    ec.echo_kv_write(pool, every, *kept)               # their scales may be smaller now
    want = host(ec.echo_kv_attention(pool, batch, q, causal_block=1))
    mass = P.attend(I.values(host(pool.pages), host(pool.scale)), None, base.table, base.lens, base.row0, host(q),
                    2, 1)[1]
    for p in (3, n - 1, n - rows):
        k, v = kept[0].clone(), kept[1].clone()
        (k, v)[kv][p, d + 32] = float(value)
        ec.echo_kv_write(pool, every, k, v)
        assert ec.echo_get_device_error() == 5
        got = host(ec.echo_kv_attention(pool, batch, q, causal_block=1))
        for r in range(rows):
            if n - rows + r >= p:
                assert not np.isfinite(got[r, d + 32:d + 64]).any()
                assert same(got[r, :d], want[r, :d])
            else:
                assert same(got[r, :d], want[r, :d])
                assert (np.abs(got[r, d:] - want[r, d:]) <= 2 * TOL * mass[r, d:] + 1e-30).all()


def test_pages_that_are_none(ec):
    for rows in (1, 60):
        c = int4_case.make(16, 1, 64, [100], [rows])
        pool, batch = c.device(ec)
        batch.table[0, 2] = 10 ** 6
        out = ec.echo_kv_attention(pool, batch, bf(kv_case.queries(rows, 64, 1)))
        assert ec.echo_get_device_error() == 8 and out.shape == (rows, 64)


def test_captured_and_replayed(ec):
    """Write, attention and read in a graph, replayed after the rows have changed."""
    import torch
    c = int4_case.make(32, 2, 128, [300, 41], [4, 41])
    pool, batch = c.device(ec)
    k, v, hk, hv = sources(c.n_rows, 256, "bf16", seed=3)
    q = bf(kv_case.queries(c.n_rows, 512, 4))
    kk, vv, qq = k.contiguous(), v.contiguous(), q.clone()
    out = torch.empty_like(q)
    ws = torch.empty(ec.echo_kv_attention_workspace_size(pool, batch, 4), dtype=torch.uint8, device="cuda")

    def step():
        ec.echo_kv_write(pool, batch, kk, vv)
        return ec.echo_kv_attention(pool, batch, qq, causal_block=1, out=out, workspace=ws)

    step()
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        step()
    for factor in (2.0, -0.5):
        kk.copy_(k * factor)
        vv.copy_(v * factor)
        g.replay()
        torch.cuda.synchronize()
        c.pages, c.scale = written(c, host(kk), host(vv))
        want, mass = P.attend(c.values, None, c.table, c.lens, c.row0, host(q), 4, 1)
        close(host(out), want, mass)
    assert ec.echo_get_device_error() == 0
