"""Refusals of the page tables', rotary positions', gated norms' and 4-bit pages' entry points: every
bad argument answers before anything reaches a GPU.  No GPU."""
import ctypes

import pytest

FAKE = 0x10000          # a 16-byte aligned address that is never dereferenced by the checks
INF, NAN = float("inf"), float("nan")


@pytest.fixture(scope="module")
def ec():
    import shutil
    import os
    if not shutil.which("nvcc") and not os.path.exists("/usr/local/cuda/bin/nvcc"):
        pytest.skip("nvcc not available")
    from paper_2608_02474_gb300 import build
    build.build()
    from paper_2608_02474_gb300 import echocache
    return echocache


def no_gpu():
    import torch
    return not torch.cuda.is_available()


TABLES = dict(n_pages=8, page_tokens=16, n_slots=4, max_pages=3, table=FAKE, len=FAKE, free_pages=FAKE, n_free=FAKE)


def tables(ec, change=None, null=False, slots=FAKE, rows=FAKE, n=2, n_rows=5, table=FAKE, lens=FAKE, row0=FAKE,
           place=FAKE, pos=FAKE, seq=FAKE):
    """Statuses of (reset, extend, shorten)."""
    L = ec.lib()
    t = None if null else ctypes.byref(ec.KVTablesC(**{**TABLES, **(change or {})}))
    return (L.echo_kv_tables_reset(t, None),
            L.echo_kv_extend(t, slots, rows, n, n_rows, table, lens, row0, place, pos, seq, None),
            L.echo_kv_shorten(t, slots, rows, n, None))


@pytest.mark.parametrize("change,status", [
    (dict(n_pages=0), 2), (dict(page_tokens=8), 2), (dict(page_tokens=48), 2), (dict(page_tokens=256), 2),
    (dict(n_slots=0), 2), (dict(n_slots=262145), 2), (dict(max_pages=0), 2), (dict(n_slots=4096, max_pages=2 ** 20), 2),
    (dict(table=0), 1), (dict(len=0), 1), (dict(free_pages=0), 1), (dict(n_free=0), 1), (dict(table=FAKE + 2), 1),
    (dict(n_free=FAKE + 1), 1)])
def test_bad_tables(ec, change, status):
    assert tables(ec, change) == (status,) * 3


def test_bad_steps(ec):
    assert tables(ec, null=True) == (1, 1, 1)
    for bad in (dict(n=-1), dict(n=8193)):
        assert tables(ec, **bad)[1:] == (2, 2)
    for bad in (dict(rows=0), dict(rows=FAKE + 2), dict(slots=FAKE + 3)):
        assert tables(ec, **bad)[1:] == (1, 1)
    assert tables(ec, n_rows=-1)[1] == 2
    for bad in (dict(lens=0), dict(row0=0), dict(table=FAKE + 1), dict(lens=FAKE + 2), dict(row0=FAKE + 2),
                dict(place=FAKE + 4), dict(pos=FAKE + 2), dict(seq=FAKE + 1)):
        assert tables(ec, **bad)[1] == 1, bad
    assert tables(ec, n=0, rows=0, slots=0)[2] == 0          # nothing to shorten
    if no_gpu():
        assert tables(ec, slots=None, table=None, place=None, pos=None, seq=None) == (7, 7, 7)


POOL = dict(kind=3, n_pages=4, page_tokens=16, H=2, d=64, pages=FAKE, scale=FAKE)


def write_at(ec, change=None, null=False, place=FAKE, n=5, k=FAKE, v=FAKE, ld=128, t=0):
    p = None if null else ctypes.byref(ec.KVPoolC(**{**POOL, **(change or {})}))
    return ec.lib().echo_kv_write_at(p, place, n, k, v, ld, t, None)


def test_write_at(ec):
    assert write_at(ec, null=True) == 1
    for change, status in ((dict(kind=2), 1), (dict(kind=4), 1), (dict(n_pages=0), 2), (dict(page_tokens=24), 2),
                           (dict(d=96), 2), (dict(H=0), 2), (dict(pages=0), 1), (dict(pages=FAKE + 8), 1),
                           (dict(scale=0), 1), (dict(scale=FAKE + 2), 1), (dict(n_pages=2 ** 30, H=1), 2)):
        assert write_at(ec, change) == status, change
    for bad, status in ((dict(place=0), 1), (dict(place=FAKE + 4), 1), (dict(n=-1), 2), (dict(k=0), 1), (dict(v=0), 1),
                        (dict(k=FAKE + 8), 1), (dict(ld=120), 2), (dict(ld=132), 2), (dict(t=2), 1)):
        assert write_at(ec, **bad) == status, bad
    assert write_at(ec, n=0, place=0, k=0, v=0) == 0
    if no_gpu():
        assert write_at(ec) == 7 and write_at(ec, dict(kind=1, scale=0)) == 7 and write_at(ec, dict(kind=0)) == 7


def test_pools_of_four_bits(ec):
    b = ctypes.byref(ec.KVBatchC(table=FAKE, len=FAKE, row0=FAKE, n_seqs=2, max_pages=3, n_rows=5, max_rows=3))
    L = ec.lib()
    for change, status in ((dict(scale=0), 1), (dict(scale=FAKE + 4), 1), (dict(d=32), 2)):
        p = ctypes.byref(ec.KVPoolC(**{**POOL, **change}))
        assert (L.echo_kv_write(p, b, FAKE, FAKE, 128, 0, None), L.echo_kv_read(p, b, FAKE, FAKE, 128, 0, None),
                L.echo_kv_attention(p, b, FAKE, 128, 2, 0, FAKE, 128, FAKE, 1 << 40, None)) == (status,) * 3
        assert L.echo_kv_attention_workspace_size(p, b, 2) == 0
    sizes = [L.echo_kv_attention_workspace_size(ctypes.byref(ec.KVPoolC(**{**POOL, "kind": k})), b, 2) for k in (0, 1, 3)]
    assert sizes[0] == sizes[1] == sizes[2] > 0
    # a cache of whole rows has no such form
    c = ec.CacheC(3, 16, 64, FAKE, FAKE, FAKE, FAKE, FAKE, FAKE, 4, 4, 0.5)
    assert L.echo_cache_reset(ctypes.byref(c), None) in (1, 2)
    assert L.echo_cache_read(ctypes.byref(c), None, 4, FAKE, None) in (1, 2)


def test_bad_turns(ec):
    def call(axes=1, pairs=(4,), theta=1e4, scaling=0, factor=1.0, original=4096.0, fast=32.0, slow=1.0, null=()):
        import numpy as np
        out, size = np.zeros(256, dtype=np.uint64), ctypes.c_float()
        prm = ec.RotaryParams(theta, scaling, factor, original, fast, slow)
        n = (ctypes.c_int32 * 4)(*pairs)
        return ec.lib().echo_rotary_turns(None if "prm" in null else ctypes.byref(prm), axes, None if "pairs" in null else n,
                                          None if "turn" in null else out.ctypes.data,
                                          None if "size" in null else ctypes.byref(size))

    assert call() == 0 and call(4, (32, 32, 32, 32)) == 0 and call(scaling=3, factor=4.0) == 0
    for name in ("prm", "pairs", "turn", "size"):
        assert call(null=(name,)) == 1
    for bad in (dict(axes=0), dict(axes=5), dict(pairs=(0,)), dict(pairs=(-1,)), dict(pairs=(129,)),
                dict(axes=2, pairs=(100, 29)), dict(axes=2, pairs=(5, -1))):
        assert call(**bad) == 2, bad
    for bad in (dict(theta=0.5), dict(theta=INF), dict(theta=NAN), dict(factor=0.5), dict(factor=INF), dict(factor=NAN),
                dict(scaling=-1), dict(scaling=4), dict(scaling=3, original=0.0), dict(scaling=3, original=NAN),
                dict(scaling=3, slow=-1.0), dict(scaling=3, fast=1.0), dict(scaling=3, fast=INF)):
        assert call(**bad) == 1, bad


ROT = dict(layout=0, axes=1, pairs=(16, 0, 0, 0), frame=0, row=0, size=1.0, turn=FAKE)


def rotary(ec, plan=None, null=False, pos=FAKE, n=3, d=64, t=0, q=FAKE, ldq=128, Hq=2, qo=FAKE, ldqo=128, k=FAKE, ldk=64,
           Hk=1, ko=FAKE, ldko=64):
    a = {**ROT, **(plan or {})}
    c = ec.RotaryPlanC(a["layout"], a["axes"], (ctypes.c_int32 * 4)(*a["pairs"]), a["frame"], a["row"], a["size"], a["turn"])
    return ec.lib().echo_rotary(None if null else ctypes.byref(c), pos, n, d, t, 0, q, ldq, Hq, qo, ldqo, k, ldk, Hk, ko,
                                ldko, None)


def test_bad_rotary(ec):
    assert rotary(ec, null=True) == 1
    for plan, status in ((dict(layout=2), 1), (dict(layout=-1), 1), (dict(size=NAN), 1), (dict(size=INF), 1),
                         (dict(axes=0), 2), (dict(axes=5), 2), (dict(pairs=(0, 9, 0, 0)), 2), (dict(pairs=(33, 0, 0, 0)), 2),
                         (dict(pairs=(-1, 0, 0, 0)), 2), (dict(axes=2, pairs=(16, 17, 0, 0)), 2), (dict(turn=0), 1),
                         (dict(turn=FAKE + 4), 1), (dict(frame=-1), 2), (dict(frame=12, row=4), 2),
                         (dict(axes=3, pairs=(4, 4, 4, 0), frame=12, row=5), 2),
                         (dict(axes=3, pairs=(4, 4, 4, 0), frame=12, row=0), 2)):
        assert rotary(ec, plan) == status, plan
    for bad, status in ((dict(t=2), 1), (dict(d=0), 2), (dict(d=60), 2), (dict(d=264), 2), (dict(n=-1), 2), (dict(Hq=0), 2),
                        (dict(Hk=-1), 2), (dict(ldq=120), 2), (dict(ldqo=132), 2), (dict(ldk=56), 2), (dict(ldko=68), 2),
                        (dict(q=0), 1), (dict(qo=0), 1), (dict(k=0), 1), (dict(ko=0), 1), (dict(q=FAKE + 8), 1),
                        (dict(qo=FAKE + 2), 1), (dict(k=FAKE + 4), 1), (dict(ko=FAKE + 8), 1), (dict(pos=0), 1),
                        (dict(pos=FAKE + 2), 1), (dict(ldqo=136), 2), (dict(ldko=72), 2)):
        assert rotary(ec, **bad) == status, bad
    assert rotary(ec, n=0, q=0, qo=0, k=0, ko=0, pos=0) == 0
    if no_gpu():
        assert rotary(ec) == 7 and rotary(ec, k=0, ko=0, Hk=0, ldk=0, ldko=0) == 7
        assert rotary(ec, ldqo=136, qo=2 * FAKE, ldko=72, ko=3 * FAKE) == 7


def gated(ec, plan=None, mod=None, null=False, n=3, x=FAKE, ldx=64, xt=0, y=2 * FAKE, ldy=64, yt=0, h=3 * FAKE, ldh=64, ht=0,
          out=4 * FAKE, ldn=64, nt=0):
    a = {**dict(D=64, after=(0, 0.0, 0, 0), before=(1, 1e-6, FAKE, FAKE), alpha=1.0, beta=1.0), **(plan or {})}
    p = ec.GatedNormPlanC(a["D"], ec.NormC(*a["after"]), ec.NormC(*a["before"]), a["alpha"], a["beta"])
    m = None
    if mod is not None:
        m = ctypes.byref(ec.ModulationC(*{**dict(gate=FAKE, scale=FAKE, shift=FAKE, ld=64, n_mods=2, per=2, rows=FAKE, t=0),
                                          **mod}.values()))
    return ec.lib().echo_gated_norm(None if null else ctypes.byref(p), m, n, x, ldx, xt, y, ldy, yt, h, ldh, ht, out, ldn,
                                    nt, None)


def test_bad_gated_norms(ec):
    assert gated(ec, null=True) == 1
    for plan, status in ((dict(D=0), 2), (dict(D=4), 2), (dict(D=60), 2), (dict(D=16392), 2), (dict(alpha=NAN), 1),
                         (dict(beta=INF), 1), (dict(before=(3, 0.0, 0, 0)), 1), (dict(after=(-1, 0.0, 0, 0)), 1),
                         (dict(before=(1, -1.0, 0, 0)), 1), (dict(before=(1, NAN, 0, 0)), 1),
                         (dict(after=(2, INF, 0, 0)), 1), (dict(before=(2, 0.0, FAKE + 8, 0)), 1),
                         (dict(before=(2, 0.0, 0, FAKE + 4)), 1), (dict(after=(0, 0.0, FAKE, 0)), 1)):
        assert gated(ec, plan) == status, plan
    for mod, status in ((dict(ld=56), 2), (dict(ld=68), 2), (dict(n_mods=-1), 2), (dict(rows=0, per=0), 2), (dict(t=2), 1),
                        (dict(gate=FAKE + 8), 1), (dict(scale=FAKE + 4), 1), (dict(shift=FAKE + 2), 1), (dict(rows=FAKE + 2), 1)):
        assert gated(ec, mod=mod) == status, mod
    for bad, status in ((dict(n=-1), 2), (dict(x=0), 1), (dict(xt=2), 1), (dict(yt=-1), 1), (dict(ht=3), 1), (dict(nt=2), 1),
                        (dict(ldx=56), 2), (dict(ldy=60), 2), (dict(ldh=8), 2), (dict(ldn=65), 2), (dict(x=FAKE + 8), 1),
                        (dict(y=FAKE + 4), 1), (dict(h=FAKE + 2), 1), (dict(out=FAKE + 8), 1),
                        (dict(h=FAKE, ht=1), 2), (dict(h=FAKE, ldh=72), 2), (dict(out=2 * FAKE, nt=1), 2),
                        (dict(out=3 * FAKE), 1)):
        assert gated(ec, **bad) == status, bad
    assert gated(ec, n=0, x=0, y=0, h=0, out=0) == 0 and gated(ec, h=0, out=0) == 0     # nothing to do
    if no_gpu():
        assert gated(ec) == 7 and gated(ec, mod={}) == 7 and gated(ec, y=0, h=0) == 7
        assert gated(ec, h=FAKE, out=2 * FAKE) == 7


def test_names(ec):
    assert [ec.echo_kernel_name(k) for k in (21, 22, 23, 24)] == ["kv_tables", "rotary", "gated_norm", "unknown"]


def test_binding_checks(ec):
    """What the binding refuses by itself: host tensors, other types and shapes."""
    import torch
    i32 = lambda *n: torch.zeros(*n, dtype=torch.int32)       # noqa: E731
    with pytest.raises(ValueError, match="CUDA"):
        ec.KVTables(i32(2, 3), i32(2), i32(4), i32(1), 16)
    with pytest.raises(TypeError):
        ec.KVTables(i32(2, 3).long(), i32(2), i32(4), i32(1), 16)
    with pytest.raises(ValueError, match="n_slots"):
        ec.KVTables(i32(6), i32(2), i32(4), i32(1), 16)
    with pytest.raises(ValueError, match="CUDA"):
        ec.KVStep(i32(2, 3), i32(2), i32(3), torch.zeros(4, dtype=torch.int64), i32(4), i32(4))
    for bad in (dict(layout="thirds"), dict(scaling="more"), dict(axis_pairs=33), dict(axis_pairs=[]), dict(axis_pairs=[1] * 5),
                dict(axis_pairs=[4, -1])):
        with pytest.raises(ValueError):
            ec.Rotary(64, **{**dict(axis_pairs=8, device="cpu"), **bad})
    with pytest.raises(ec.EchoError, match="INVALID"):
        ec.Rotary(64, 8, theta=0.1, device="cpu")
    plan = ec.Rotary(64, [8, 4], scaling="yarn", factor=4.0, original=100.0, device="cpu")
    assert plan.pairs == 12 and plan.columns == 2 and plan.turn.shape == (12,)
    x = torch.zeros(4, 128, dtype=torch.bfloat16)
    with pytest.raises(ValueError, match="CUDA"):
        ec.echo_rotary(plan, i32(4, 2), x)
    with pytest.raises(ValueError):
        ec.echo_rotary(plan, i32(4, 2), x[:, :100])
    for bad in (dict(before="batch"), dict(after="l2")):
        with pytest.raises(ValueError):
            ec.GatedNorm(64, **bad)
    with pytest.raises(ValueError, match="CUDA"):
        ec.GatedNorm(64, weight=torch.ones(64))
    with pytest.raises(ValueError, match="CUDA"):
        ec.echo_gated_norm(ec.GatedNorm(128), x)
    with pytest.raises(ValueError, match="INT4|4 bits|CUDA"):
        ec.KVPool(torch.zeros(1, 2, 1, 16, 32, dtype=torch.uint8))


def test_turns_are_the_frequencies(ec):
    """The table of turns against fp64: whole numbers of 2^-64 turns a position, cut off (an absolute
    error of up to 2^-64), from powers, quotients and sums of a few fp64 roundings on either side (2^-50 of the frequency)."""
    import numpy as np
    from oracle import rotary as R
    for scaling, factor in (("none", 1.0), ("linear", 3.0), ("ntk", 5.0), ("yarn", 7.0)):
        plan = ec.Rotary(128, [20, 0, 1, 43], theta=5e5, scaling=scaling, factor=factor, original=8192.0, device="cpu")
        freq, size = R.frequencies([20, 0, 1, 43], 5e5, scaling, factor, 8192.0)
        turn = plan.turn.numpy().view(np.uint64).astype(np.float64) / 2.0 ** 64
        want = freq / (2 * np.pi)
        assert (np.abs(turn - want) <= 2.0 ** -63 + 2.0 ** -50 * want).all() and abs(plan.size - size) < 1e-6
