"""Writing rows into the paged key/value cache and reading them back, against the oracle:
codes, scales and values bit for bit, and every other slot of the pool untouched."""
import numpy as np
import pytest

pytestmark = pytest.mark.gpu

import kv_case                                     # noqa: E402
from oracle import cache as C                      # noqa: E402
from oracle import paged as P                      # noqa: E402

F32 = np.float32


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


def sources(n, cols, dtype, seed, device=True):
    """k and v as the two halves of one wider tensor, and their host values."""
    import torch
    x = np.random.default_rng(seed).standard_normal((n, 2 * cols)).astype(F32)
    x[:, ::7] *= 8
    if n > 1:
        x[1, :cols // 2] = 0                        # a head of zeros
    t = torch.from_numpy(x).cuda().to(torch.bfloat16 if dtype == "bf16" else torch.float32)
    k, v = t[:, :cols], t[:, cols:]
    return k, v, host(k), host(v)


CASES = [
    # form, page, H, d, lens, rows
    ("int8", 16, 1, 64, [1], [1]),
    ("bf16", 16, 1, 64, [1], [1]),
    ("int8", 64, 40, 128, [200], [65]),
    ("bf16", 128, 5, 128, [129, 0, 128, 300], [129, 0, 1, 77]),
    ("int8", 32, 16, 64, [33, 31, 1000], [2, 31, 500]),
    ("int8", 16, 3, 128, list(range(1, 70)), [1] * 69),
    ("bf16", 16, 2, 64, [5] * 1100, [(b % 3) for b in range(1100)]),
    ("int8", 128, 7, 64, [260, 40], [0, 40]),
]


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("form,page,H,d,lens,rows", CASES)
def test_write(ec, form, page, H, d, lens, rows, dtype):
    c = kv_case.make(form, page, H, d, lens, rows)
    pool, batch = c.device(ec)
    k, v, hk, hv = sources(c.n_rows, H * d, dtype, seed=page + H)
    ec.echo_kv_write(pool, batch, k, v)
    assert not P.write(c.pages, c.scale, c.table, c.lens, c.row0, hk, hv)
    assert same(host(pool.pages), c.pages)
    if form == "int8":
        assert same(host(pool.scale), c.scale)
    assert ec.echo_get_device_error() == 0


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("form,page,H,d,lens,rows", CASES)
def test_read(ec, form, page, H, d, lens, rows, dtype):
    import torch
    c = kv_case.make(form, page, H, d, lens, rows, seed=1)
    pool, batch = c.device(ec)
    t = torch.bfloat16 if dtype == "bf16" else torch.float32
    want = P.read(c.pages, c.scale, c.table, c.lens, c.row0, c.n_rows)
    wide = torch.full((c.n_rows, 2 * H * d + 8), 3.0, dtype=t, device="cuda")
    ec.echo_kv_read(pool, batch, k=wide[:, :H * d], v=wide[:, H * d:2 * H * d])
    for got, w in zip(ec.echo_kv_read(pool, batch, dtype=t), want):
        assert same(host(got), C.round_bf16(w) if dtype == "bf16" else w)
    assert torch.equal(wide[:, :2 * H * d], torch.cat(ec.echo_kv_read(pool, batch, dtype=t), dim=1))
    assert bool((wide[:, 2 * H * d:] == 3.0).all())          # columns beyond are not touched
    assert ec.echo_get_device_error() == 0


@pytest.mark.parametrize("form", ["bf16", "int8"])
def test_rows_before_the_start_and_past_the_last_sequence(ec, form):
    """Positions below 0 are left out of a write and read as zeros; rows at or past
    row0[n_seqs] are not touched."""
    import torch
    c = kv_case.make(form, 16, 2, 64, [3], [5])
    pool, batch = c.device(ec)
    batch = ec.KVBatch(batch.table, batch.lens, batch.row0, 7)
    k, v, hk, hv = sources(7, 128, "f32", seed=4)
    ec.echo_kv_write(pool, batch, k, v)
    P.write(c.pages, c.scale, c.table, c.lens, c.row0, hk, hv)
    assert same(host(pool.pages), c.pages)
    out = [torch.full((7, 128), 9.0, device="cuda") for _ in range(2)]
    ec.echo_kv_read(pool, batch, k=out[0], v=out[1])
    for got, w in zip(out, P.read(c.pages, c.scale, c.table, c.lens, c.row0, 7)):
        w[5:] = 9.0
        assert same(host(got), w) and not w[:2].any()
    assert ec.echo_get_device_error() == 0


@pytest.mark.parametrize("value", [np.inf, -np.inf, np.nan])
def test_non_finite_rows(ec, value):
    """INT8: codes 0, the |maximum| as the scale, the device flag; other heads unharmed.
    BF16 pages keep the value."""
    c = kv_case.make("int8", 16, 3, 64, [20], [4])
    pool, batch = c.device(ec)
    k, v, hk, hv = sources(4, 192, "f32", seed=5)
    k[2, 64 + 9], hk[2, 64 + 9] = float(value), value
    ec.echo_kv_write(pool, batch, k, v)
    assert P.write(c.pages, c.scale, c.table, c.lens, c.row0, hk, hv)
    assert same(host(pool.pages), c.pages) and same(host(pool.scale), c.scale)
    assert ec.echo_get_device_error() == 5
    c = kv_case.make("bf16", 16, 3, 64, [20], [4])
    pool, batch = c.device(ec)
    ec.echo_kv_write(pool, batch, k, v)
    P.write(c.pages, c.scale, c.table, c.lens, c.row0, hk, hv)
    assert same(host(pool.pages), c.pages)
    assert ec.echo_get_device_error() == 0


@pytest.mark.parametrize("form", ["bf16", "int8"])
def test_table_entries_outside_the_pool(ec, form):
    """A page number that is none, and a length past the table: the flag, the other rows
    written and read as ever, the rows in question left out and read as zeros."""
    c = kv_case.make(form, 16, 1, 64, [40, 40], [40, 40])
    for page in (-1, c.pages.shape[0], 2 ** 31 - 1, -2 ** 31):
        pool, batch = c.device(ec)
        before = pool.pages.clone()
        batch.table[0, 1] = page
        k, v, hk, hv = sources(80, 64, "bf16", seed=6)
        ec.echo_kv_write(pool, batch, k, v)
        assert ec.echo_get_device_error() == 8
        want = host(before)
        P.write(want, None if c.scale is None else c.scale.copy(), c.table, c.lens, c.row0, hk, hv)
        want[c.table[0, 1]] = host(before)[c.table[0, 1]]
        assert same(host(pool.pages), want)
        got, _ = ec.echo_kv_read(pool, batch)
        assert ec.echo_get_device_error() == 8
        assert not got[16:32].any() and bool(got[:16].any(dim=1).all())
    pool, batch = c.device(ec)
    batch.lens[1] = 57                               # 17 rows past the table's 48 positions
    got, _ = ec.echo_kv_read(pool, batch)
    assert ec.echo_get_device_error() == 8
    assert not got[40 + 31:].any()


def test_another_stream_and_empty_calls(ec):
    import torch
    c = kv_case.make("int8", 32, 4, 128, [100], [100])
    pool, batch = c.device(ec)
    k, v, hk, hv = sources(100, 512, "bf16", seed=8)
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    ec.echo_kv_write(pool, batch, k, v, stream=s)
    got = ec.echo_kv_read(pool, batch, stream=s)
    s.synchronize()
    P.write(c.pages, c.scale, c.table, c.lens, c.row0, hk, hv)
    for g, w in zip(got, P.read(c.pages, c.scale, c.table, c.lens, c.row0, 100)):
        assert same(host(g), C.round_bf16(w))
    n = ec.echo_launch_count()
    none = ec.KVBatch(batch.table[:0], batch.lens[:0], batch.row0[:1], 0)
    ec.echo_kv_write(pool, none, k[:0], v[:0])
    ec.echo_kv_read(pool, none)
    assert ec.echo_launch_count() == n and ec.echo_get_device_error() == 0


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_heads_of_the_smallest_values(ec, dtype):
    """Below 127 / FLT_MAX (3.7e-37) 127 / a is infinite in fp32, and the rule's clamp gives
    +-127 to every value but 0, which stays 0."""
    import torch
    largest = [1e-36, 3.8e-37, 3.7e-37, 1e-37, 1.2e-38, 3e-39, 1e-40, 1.0]
    H, d, n = len(largest), 64, 5
    x = np.random.default_rng(9).uniform(-1, 1, (n, H, d)) * np.array(largest)[:, None]
    x[:, :, 3] = largest
    x[:, :, 10:14], x[:, :, 11] = 0, -0.0
    t = torch.from_numpy(x.astype(F32).reshape(n, H * d)).cuda()
    k = t.to(torch.bfloat16) if dtype == "bf16" else t
    c = kv_case.make("int8", 16, H, d, [n], [n])
    pool, batch = c.device(ec)
    ec.echo_kv_write(pool, batch, k, -k)
    v = host(k).reshape(n, H, d)
    a = np.abs(v).max(axis=2, keepdims=True)
    with np.errstate(over="ignore", invalid="ignore"):
        inv = F32(127) / a
        q = np.where(v == 0, 0, np.clip(np.rint(v * inv), -127, 127)).astype(np.int8)
    assert np.isinf(inv[:, 2:7]).all() and np.isfinite(inv[:, :2]).all()
    assert (np.abs(q[:, 2:7]) == np.where(v[:, 2:7] == 0, 0, 127)).all()
    page = c.table[0, 0]
    for i, codes in ((0, q), (1, -q)):
        assert same(host(pool.pages)[page, i, :, :n].transpose(1, 0, 2), codes)
        assert same(host(pool.scale)[page, i, :, :n].T, (a / F32(127))[..., 0])
    back, _ = ec.echo_kv_read(pool, batch, dtype=torch.float32)
    assert same(host(back).reshape(n, H, d), q.astype(F32) * (a / F32(127)))
    assert ec.echo_get_device_error() == 0
