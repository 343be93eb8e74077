"""Tables that are wider than their sequences need: the work is divided by the longest sequence
that the host tells of, and the results are right whatever it tells.  Tolerance of
test_gpu_kv_attention.py."""
import numpy as np
import pytest

pytestmark = pytest.mark.gpu

import int4_case                                   # noqa: E402
import kv_case                                     # noqa: E402
from oracle import paged as P                      # noqa: E402
from synth import generate as G                    # noqa: E402
from test_gpu_chunk_stream_device import F32, W, bf, cond_kv   # noqa: E402

TOL = 2.15 * 2.0 ** -8
FORMS = pytest.mark.parametrize("form", ["bf16", "int8", "int4"])


@pytest.fixture(scope="module")
def ec():
    import torch
    if not torch.cuda.is_available():
        pytest.skip("needs a GPU")
    from paper_2608_02474_gb300 import echocache
    return echocache


def make(form, *a, **kw):
    return int4_case.make(*a, **kw) if form == "int4" else kv_case.make(form, *a, **kw)


@FORMS
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("rows", [1, 100])
def test_as_over_a_table_of_its_own_width(ec, form, d, rows):
    import torch
    c = make(form, 64, 2, d, [700, 300], [rows, 1], seed=rows)
    q = kv_case.queries(c.n_rows, 2 * d, 3, 1.5)
    pool, batch = c.device(ec)
    table = torch.full((2, 8192), -1, dtype=torch.int32, device="cuda")
    table[:, :c.table.shape[1]] = batch.table

    def run(b):
        n = ec.echo_launch_count()
        out = ec.echo_kv_attention(pool, b, bf(q), causal_block=1)
        return out, ec.echo_launch_count() - n

    own, launches = run(batch)
    assert launches == 1
    far = lambda n: ec.KVBatch(table, batch.lens, batch.row0, c.n_rows, rows, n)   # noqa: E731
    for n in (700, 704, 641):                       # whole pages of the longest
        out, launches = run(far(n))
        assert launches == 1 and (out == own).all(), n
    pages, scale = (c.values, None) if form == "int4" else (c.pages, c.scale)
    want, mass = P.attend(pages, scale, c.table, c.lens, c.row0, q, 2, 1)
    for n in (None, 1, 10 ** 5, 2 ** 31 - 1):
        out, launches = run(far(n))
        assert launches == (1 if n == 1 else 2)
        assert (np.abs(out.float().cpu().numpy() - want) <= TOL * mass + 1e-30).all(), n
    assert ec.echo_get_device_error() == 0


@FORMS
@pytest.mark.parametrize("rows", [1, 40])
def test_long_sequences_told_to_be_short(ec, form, rows):
    """Not divided then, but right."""
    c = make(form, 32, 2, 64, [5000, 20], [rows, 2], seed=1)
    q = kv_case.queries(c.n_rows, 128, 3, 1.5)
    pool, batch = c.device(ec)
    batch.max_len = 20
    out = ec.echo_kv_attention(pool, batch, bf(q), causal_block=1).float().cpu().numpy()
    pages, scale = (c.values, None) if form == "int4" else (c.pages, c.scale)
    want, mass = P.attend(pages, scale, c.table, c.lens, c.row0, q, 2, 1)
    assert (np.abs(out - want) <= TOL * mass + 1e-30).all() and ec.echo_get_device_error() == 0


@FORMS
def test_launches_of_a_chunk_stream(ec, form):
    """Short clips in large pools: attention is not divided, whoever keeps the tables."""
    from paper_2608_02474_gb300.pipeline import ChunkStream
    kind = {"bf16": ec.CACHE_BF16, "int8": ec.CACHE_INT8, "int4": ec.CACHE_INT4}[form]
    weights = [G.block_weights(W, l) for l in range(2)]
    kv = cond_kv(ec, weights, G.random_rows(672, W.D, seed=3))
    for device_tables in (False, True):
        st = ChunkStream([ec.DeviceBlock.from_host(w, np.zeros((1, W.D), F32)) for w in weights], W.H, W.d, 24,
                         n_pages=4096, cond_pages=64, kind=kind, device_tables=device_tables)
        st.open(0, kv)
        st.step({0: bf(G.random_rows(24, W.D, seed=4))})
        ec.echo_profile_enable(True)
        ec.echo_profile_read()
        st.step({0: bf(G.random_rows(1, W.D, seed=5))})
        names = [r[0] for r in ec.echo_profile_read()]
        ec.echo_profile_enable(False)
        assert names.count("kv_attention") == 4 and "kv_join" not in names, (device_tables, names)
    assert ec.echo_get_device_error() == 0
