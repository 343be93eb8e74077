"""Refusals of the paged key/value cache's entry points: every bad argument answers before
anything reaches a GPU.  No GPU."""
import ctypes
import os

import pytest

FAKE = 0x10000          # a 16-byte aligned address that is never dereferenced by the checks


@pytest.fixture(scope="module")
def ec():
    import shutil
    if not shutil.which("nvcc") and not os.path.exists("/usr/local/cuda/bin/nvcc"):
        pytest.skip("nvcc not available")
    from paper_2608_02474_gb300 import build
    build.build()
    from paper_2608_02474_gb300 import echocache
    return echocache


POOL = dict(kind=0, n_pages=4, page_tokens=16, H=2, d=64, pages=FAKE, scale=FAKE)
BATCH = dict(table=FAKE, len=FAKE, row0=FAKE, n_seqs=2, max_pages=3, n_rows=5, max_rows=3)

BAD_POOLS = [
    (dict(kind=2), 1), (dict(kind=-1), 1), (dict(n_pages=0), 2), (dict(page_tokens=0), 2),
    (dict(page_tokens=24), 2), (dict(page_tokens=256), 2), (dict(H=0), 2), (dict(d=32), 2),
    (dict(d=96), 2), (dict(pages=0), 1), (dict(pages=FAKE + 8), 1), (dict(scale=0), 1),
    (dict(scale=FAKE + 4), 1), (dict(n_pages=2 ** 30, H=1), 2),
]
BAD_BATCHES = [
    (dict(n_seqs=-1), 2), (dict(max_pages=-1), 2), (dict(n_rows=-1), 2), (dict(max_rows=-1), 2),
    (dict(len=0), 1), (dict(row0=0), 1), (dict(table=0), 1), (dict(table=FAKE + 2), 1),
    (dict(len=FAKE + 1), 1), (dict(row0=FAKE + 3), 1),
]


def calls(ec, pool=None, batch=None, x=FAKE, ld=128, t=0, Hq=2, cb=0, out=FAKE, ldo=128, ws=FAKE,
          wsb=1 << 40, null=(), which=(0, 1, 2)):
    """Statuses of (write, read, attention), or of `which` of them: only calls that the checks
    refuse, since the addresses are not real and a machine may have a GPU."""
    L = ec.lib()
    p = ec.KVPoolC(**{**POOL, **(pool or {})})
    b = ec.KVBatchC(**{**BATCH, **(batch or {})})
    p, b = (None if "pool" in null else ctypes.byref(p)), (None if "batch" in null else ctypes.byref(b))
    make = (lambda: L.echo_kv_write(p, b, x, FAKE, ld, t, None), lambda: L.echo_kv_read(p, b, FAKE, x, ld, t, None),
            lambda: L.echo_kv_attention(p, b, x, ld, Hq, cb, out, ldo, ws, wsb, None))
    return tuple(make[i]() for i in which)


@pytest.mark.parametrize("change,status", BAD_POOLS)
def test_bad_pools(ec, change, status):
    assert calls(ec, pool=change) == (status,) * 3
    p, b = ec.KVPoolC(**{**POOL, **change}), ec.KVBatchC(**BATCH)
    assert ec.lib().echo_kv_attention_workspace_size(ctypes.byref(p), ctypes.byref(b), 2) == 0


@pytest.mark.parametrize("change,status", BAD_BATCHES)
def test_bad_batches(ec, change, status):
    assert calls(ec, batch=change) == (status,) * 3


def test_bad_tensors(ec):
    assert calls(ec, null=("pool",)) == (1, 1, 1) and calls(ec, null=("batch",)) == (1, 1, 1)
    assert calls(ec, x=0) == (1, 1, 1) and calls(ec, x=FAKE + 8) == (1, 1, 1)
    assert calls(ec, ld=120) == (2, 2, 2) and calls(ec, ld=132) == (2, 2, 2)
    assert calls(ec, t=2, which=(0, 1)) == (1, 1)
    for bad in (dict(Hq=0), dict(Hq=1), dict(Hq=3, ld=192, ldo=192), dict(Hq=258, ld=1 << 15, ldo=1 << 15),
                dict(cb=-1), dict(ldo=120), dict(ldo=130), dict(Hq=-2)):
        assert calls(ec, **bad, which=(2,)) == (2,), bad
    for bad in (dict(out=0), dict(out=FAKE + 4), dict(ws=0), dict(ws=FAKE + 16)):
        assert calls(ec, **bad, which=(2,)) == (1,), bad
    p, b = ec.KVPoolC(**POOL), ec.KVBatchC(**BATCH)
    need = ec.lib().echo_kv_attention_workspace_size(ctypes.byref(p), ctypes.byref(b), 2)
    assert need > 0 and calls(ec, wsb=need - 1, which=(2,)) == (3,)


def test_empty_calls_are_fine(ec):
    """No sequences or no rows: nothing to do, whatever the pointers."""
    none = dict(table=0, len=0, row0=0)
    assert calls(ec, batch=dict(n_seqs=0, **none), x=0) == (0, 0, 0)
    assert calls(ec, batch=dict(n_rows=0, **none), x=0) == (0, 0, 0)
    assert calls(ec, batch=dict(n_rows=0), pool=dict(d=32)) == (2, 2, 2)      # but sizes are checked


def test_a_bf16_pool_has_no_scale(ec):
    """kind BF16 ignores scale: the call passes the checks and stops at the missing GPU."""
    import torch
    if torch.cuda.is_available():
        pytest.skip("the addresses are not real")
    assert calls(ec, pool=dict(kind=1, scale=0)) == (7, 7, 7)


def test_names(ec):
    assert ec.status_str(8) == "ECHO_ERR_PAGE"
    assert [ec.echo_kernel_name(k) for k in (17, 18, 19)] == ["kv_write", "kv_read", "kv_attention"]


def test_binding_checks(ec):
    """What the binding refuses by itself: host tensors, other types and shapes."""
    import torch
    with pytest.raises(ValueError, match="CUDA"):
        ec.KVPool(torch.zeros(1, 2, 1, 16, 64, dtype=torch.int8))
    with pytest.raises(ValueError, match="CUDA"):
        ec.KVBatch(torch.zeros(1, 1, dtype=torch.int32), torch.zeros(1, dtype=torch.int32),
                   torch.zeros(2, dtype=torch.int32), 1)
    with pytest.raises(ValueError, match="INT8 or"):
        ec.KVPool.empty(ec.CACHE_REF, 1, 16, 1, 64)


def test_workspace_size_of_sizes_that_the_attention_refuses(ec):
    def size(Hq, **batch):
        p, b = ec.KVPoolC(**POOL), ec.KVBatchC(**{**BATCH, **batch})
        return ec.lib().echo_kv_attention_workspace_size(ctypes.byref(p), ctypes.byref(b), Hq)

    assert size(2) > 0 and size(256) > 0 and size(0, n_seqs=0) == 0
    assert [size(Hq) for Hq in (-2, 0, 1, 3, 258)] == [0] * 5
    assert size(2, n_rows=2 ** 30 - 1) > 0 and size(2, n_rows=2 ** 30) == 0
