"""ChunkStream with its page tables on the GPU, rotary positions, modulations and 4-bit pages,
against the oracle's parts over the whole clip in fp64; and such a step in a graph.

Tolerances: those of the block step (max 2e-2 normwise per token, mean 5e-3).  Pages of codes add a
quantisation error: the oracle quantises its own keys and values by the same rule, from values that differ by
the block's own errors.  A key or value near the middle between two codes may then take the other one: an
error of a step, for the few that lie so near.  int8 steps are 1 / 127 of a head's largest value and stay within the
same bars; a 4-bit step is 1 / 7 of a group's largest value, up to 1 / 5 of a typical value, and values that are off
by 2^-8 of themselves (their own rounding to bf16, and their sum's) lie that near in about 2^-8 * 5 = 2 % of the cases: a relative
error of sqrt(0.02) * 0.2 = 3 % of a key or value where they are few, averaged by the attention; the bars are doubled.
"""
import numpy as np
import pytest

pytestmark = pytest.mark.gpu

import oracle                                      # noqa: E402
from oracle import int4 as I4                      # noqa: E402
from oracle import norms, rotary                   # noqa: E402
from synth import TINY_256, generate as G          # noqa: E402

F32 = np.float32
W = TINY_256
PAIRS, GRID = [12, 10, 10], (24, 6)


@pytest.fixture(scope="module")
def ec():
    import torch
    if not torch.cuda.is_available():
        pytest.skip("needs a GPU")
    from paper_2608_02474_gb300 import echocache
    return echocache


def stored(x, H, form):
    """Keys or values as the pages hold them."""
    r = oracle.cache.round_bf16(x.astype(F32))
    if form == "bf16":
        return r
    d = x.shape[1] // H
    out = []
    for h in range(H):
        part = r[:, h * d:(h + 1) * d]
        if form == "int8":
            q, s, _ = oracle.cache.quantize_rows(part)
            out.append(q.astype(np.float64) * s[:, None])
        else:
            q, s, _ = I4.quantize(part)
            out.append(q.astype(np.float64) * np.repeat(s.astype(np.float64), 32, axis=1))
    return np.concatenate(out, axis=1)


def attend(Q, K, V, H, tops, form):
    K, V = stored(K, H, form), stored(V, H, form)
    out = np.zeros_like(Q)
    for i, n in enumerate(tops):
        out[i] = oracle.block.mha(Q[i:i + 1], K[:n], V[:n], H)[0]
    return out


def reference(x, weights, conds, frame, form, turned, mods):
    B, n = oracle.block, x.shape[0]
    tops = [min(n, (p // frame + 1) * frame) for p in range(n)]
    freq, _ = rotary.frequencies(PAIRS, 10000.0)
    turn = lambda a: rotary.turn(a, np.arange(n), W.d, PAIRS, freq, frame=GRID)[0] if turned else a   # noqa: E731
    for l, (w, cond) in enumerate(zip(weights, conds)):
        sa, ca, ga, sf, cf, gf = mods[l].astype(np.float64) if mods is not None else (0, 0, 1, 0, 0, 1)
        lin = lambda a, m: B.linear(a, w["W" + m], w["b" + m])     # noqa: E731
        x = x.astype(np.float64)
        n1 = norms.norm(x, "layer") * (1 + ca) + sa
        h1 = x + ga * lin(attend(turn(lin(n1, "q")), turn(lin(n1, "k")), lin(n1, "v"), W.H, tops, form), "o")
        kc, vc = B.cross_kv(cond, w)
        h2 = h1 + lin(attend(lin(B.layer_norm(h1), "qc"), kc, vc, W.H, [len(cond)] * n, form), "oc")
        nf = norms.norm(h2, "layer") * (1 + cf) + sf
        x = oracle.cache.round_bf16((h2 + gf * B.linear(B.gelu_tanh(B.linear(nf, w["W1"], w["b1"])), w["W2"], w["b2"]))
                                    .astype(F32))
    return x


def bf(a):
    import torch
    return torch.from_numpy(np.ascontiguousarray(a)).to("cuda", torch.bfloat16)


def cond_kv(ec, weights, cond):
    import torch
    return [ec.echo_precompute_cross_kv(bf(cond), torch.cat([bf(w["Wkc"]), bf(w["Wvc"])]),
                                        torch.cat([bf(w["bkc"]), bf(w["bvc"])])) for w in weights]


@pytest.mark.parametrize("form", ["bf16", "int8", "int4"])
@pytest.mark.parametrize("turned,modulated", [(False, False), (True, False), (False, True), (True, True)])
def test_several_clips(ec, form, turned, modulated):
    import torch
    from paper_2608_02474_gb300.pipeline import ChunkStream
    g = np.random.default_rng(7)
    weights = [G.block_weights(W, l) for l in range(2)]
    conds = {c: G.random_rows(n, W.D, seed=40 + c) for c, n in ((0, 32), (1, 7), (2, 90))}
    total = {0: 120, 1: 72, 2: 96}
    xs = {c: G.random_rows(n, W.D, seed=50 + c) for c, n in total.items()}
    mods = {c: (g.standard_normal((2, 6, W.D)) * 0.3).astype(F32) for c in total} if modulated else None
    for m in (mods or {}).values():
        m[:, [2, 5]] += 1
    kind = {"bf16": ec.CACHE_BF16, "int8": ec.CACHE_INT8, "int4": ec.CACHE_INT4}[form]
    st = ChunkStream([ec.DeviceBlock.from_host(w, np.zeros((1, W.D), F32)) for w in weights], W.H, W.d, 24, n_pages=14,
                     cond_pages=8, page_tokens=16, kind=kind, device_tables=True, max_clips=2,
                     rotary=ec.Rotary(W.d, PAIRS, frame=GRID) if turned else None)
    got, at = {c: [] for c in total}, dict.fromkeys(total, 0)

    def step(lengths):
        m = None if mods is None else {c: torch.from_numpy(mods[c]).cuda() for c in lengths}
        y = st.step({c: bf(xs[c][at[c]:at[c] + n]) for c, n in lengths.items()}, m)
        for c, n in lengths.items():
            got[c].append(y[c].float().cpu().numpy())
            at[c] += n

    st.open(0, cond_kv(ec, weights, conds[0]))
    st.open(1, cond_kv(ec, weights, conds[1]))
    with pytest.raises(MemoryError):
        st.open(2, cond_kv(ec, weights, conds[2]))     # no slot
    step({0: 24, 1: 24})
    step({0: 24})
    with pytest.raises(MemoryError):
        st.step({0: bf(np.zeros((140, W.D), F32)), 1: bf(np.zeros((140, W.D), F32))})
    step({1: 48, 0: 24})
    st.close(1)
    st.open(2, cond_kv(ec, weights, conds[2]))
    step({2: 24, 0: 48})
    st.close(0)
    step({2: 72})
    st.close(2)
    assert ec.echo_get_device_error() == 0
    for t, n in ((st.self_table, 14), (st.cond_table, 8)):
        assert t.n_free == n and t.tables.n_free.tolist() == [n] and sorted(t.tables.free_pages.tolist()) == list(range(n))
        assert not t.tables.lens.any() and not t.slots
    bar = 2 if form == "int4" else 1
    for c in total:
        y = np.concatenate(got[c])
        cond = [G.to_bf16_values(conds[c])] * 2
        ref = reference(G.to_bf16_values(xs[c]), weights, cond, 24, form, turned, None if mods is None else mods[c])
        rel = np.abs(y - ref).max(axis=1) / np.abs(ref).max(axis=1)
        mean = np.abs(y - ref).sum() / np.abs(ref).sum()
        assert rel.max() <= bar * 2e-2 and mean <= bar * 5e-3, (c, rel.max(), mean)


def test_the_same_as_with_tables_on_the_host(ec):
    """Plain blocks: both bookkeepings within the sums' order of one another."""
    from paper_2608_02474_gb300.pipeline import ChunkStream
    weights = [G.block_weights(W, l) for l in range(2)]
    kv = cond_kv(ec, weights, G.random_rows(20, W.D, seed=3))
    x = G.random_rows(60, W.D, seed=4)
    out = []
    for device_tables in (False, True):
        st = ChunkStream([ec.DeviceBlock.from_host(w, np.zeros((1, W.D), F32)) for w in weights], W.H, W.d, 1, n_pages=6,
                         cond_pages=2, page_tokens=16, device_tables=device_tables)
        st.open(5, kv)
        out.append(np.concatenate([st.step({5: bf(x[lo:lo + 20])})[5].float().cpu().numpy() for lo in (0, 20, 40)]))
    assert np.abs(out[0] - out[1]).max() <= 2e-2 * np.abs(out[0]).max() and ec.echo_get_device_error() == 0


def test_refusals_leave_the_clips(ec):
    import torch
    from paper_2608_02474_gb300.pipeline import ChunkStream
    w = G.block_weights(W, 0)
    blocks = [ec.DeviceBlock.from_host(w, np.zeros((1, W.D), F32))]
    with pytest.raises(ValueError, match="device_tables"):
        ChunkStream(blocks, W.H, W.d, 1, 4, 2, rotary=ec.Rotary(W.d, 8))
    with pytest.raises(ValueError):
        ChunkStream(blocks, W.H, W.d, 1, 4, 2, device_tables=True, rotary=ec.Rotary(W.d, [4, 4]))
    host = ChunkStream(blocks, W.H, W.d, 1, 4, 2)
    kv = cond_kv(ec, [w], G.random_rows(4, W.D, seed=1))
    host.open(0, kv)
    mod = torch.zeros(1, 6, W.D, device="cuda")
    with pytest.raises(ValueError, match="device_tables"):
        host.step({0: bf(np.zeros((1, W.D), F32))}, {0: mod})
    st = ChunkStream(blocks, W.H, W.d, 1, 4, 2, device_tables=True)
    st.open(0, kv)
    with pytest.raises(ValueError, match="open already"):
        st.open(0, kv)
    for bad in ({}, {0: mod[:, :5]}, {1: mod}):
        with pytest.raises(ValueError, match="modulations"):
            st.step({0: bf(np.zeros((1, W.D), F32))}, bad)
    with pytest.raises(ValueError):
        st.step({0: bf(np.zeros((3, W.D), F32))}, {0: mod.cpu()})     # fails inside: the step is taken back
    assert st.self_table.lens == {0: 0} and st.self_table.tables.lens.tolist()[:1] == [0]
    assert st.self_table.n_free == 4 and st.self_table.tables.n_free.tolist() == [4]
    assert st.step({0: bf(np.zeros((0, W.D), F32))})[0].shape == (0, W.D)
    st.step({0: bf(np.ones((3, W.D), F32))}, {0: mod})
    assert st.self_table.tables.lens.tolist()[:1] == [3] and ec.echo_get_device_error() == 0


@pytest.mark.parametrize("form", ["int4", "int8", "bf16"])
def test_a_step_in_a_graph(ec, form):
    """Tables, norm, projections, turns, pages and attention in one graph, replayed over page borders: the
    same numbers as the calls one by one; and two graphs that share the tables and the workspace."""
    import torch
    H, d, D, B = 2, 64, 128, 3
    w = G.block_weights(W, 0)
    kind = {"bf16": ec.CACHE_BF16, "int8": ec.CACHE_INT8, "int4": ec.CACHE_INT4}[form]
    Wq, bq, Wkv, bkv = bf(w["Wq"]), bf(w["bq"]), torch.cat([bf(w["Wk"]), bf(w["Wv"])]), torch.cat([bf(w["bk"]), bf(w["bv"])])
    plan, norm = ec.Rotary(d, 32, layout="halves"), ec.GatedNorm(D)
    mods = torch.randn(B, 3 * D, generator=torch.Generator("cuda").manual_seed(1), device="cuda") * 0.2

    class Side:
        def __init__(self):
            self.pool, self.tables = ec.KVPool.empty(kind, 24, 16, H, d), ec.KVTables.empty(24, 16, B, 8)
            self.step = ec.KVStep.empty(self.tables, B, 5, 2)
            self.x, self.h = torch.zeros(5, D, device="cuda"), torch.zeros(5, D, device="cuda")
            self.y, self.out = (torch.zeros(5, D, dtype=torch.bfloat16, device="cuda") for _ in range(2))
            self.n = torch.zeros(5, D, dtype=torch.bfloat16, device="cuda")
            self.rows = torch.tensor([1, 2, 1], dtype=torch.int32, device="cuda")
            self.ws = torch.empty(ec.echo_kv_attention_workspace_size(self.pool, self.step.batch, H), dtype=torch.uint8,
                                  device="cuda")
            self.q = torch.zeros(5, D, dtype=torch.bfloat16, device="cuda")
            self.kv = torch.zeros(5, 2 * D, dtype=torch.bfloat16, device="cuda")

        def run(self):
            ec.echo_kv_extend(self.tables, self.rows, self.step)
            ec.echo_gated_norm(norm, self.x, self.y, mods[:, :D], mods[:, D:2 * D], mods[:, 2 * D:], mod_rows=self.step.seq,
                               h=self.h, n=self.n)
            ec.echo_linear(self.n, Wq, bq, out=self.q)
            ec.echo_linear(self.n, Wkv, bkv, out=self.kv)
            ec.echo_rotary(plan, self.step.pos, self.q, self.kv[:, :D], q_out=self.q, k_out=self.kv[:, :D])
            ec.echo_kv_write_at(self.pool, self.step.place, self.kv[:, :D], self.kv[:, D:])
            ec.echo_kv_attention(self.pool, self.step.batch, self.q, causal_block=1, out=self.out, workspace=self.ws)

        def back(self):
            ec.echo_kv_shorten(self.tables, self.rows)

    a, b = Side(), Side()
    for s in (a, b):                                    # warm up, and begin again
        s.run()
        s.tables.reset()
    torch.cuda.synchronize()
    g, g2, undo = (torch.cuda.CUDAGraph() for _ in range(3))
    with torch.cuda.graph(g):
        a.run()
    with torch.cuda.graph(g2):
        a.run()
    with torch.cuda.graph(undo):
        a.back()
    for i in range(40):
        for s in (a, b):
            torch.manual_seed(i)
            s.x.copy_(torch.randn(5, D, device="cuda"))
            s.y.copy_(torch.randn(5, D, device="cuda"))
            s.out.fill_(7.0)
            s.h.fill_(7.0)
        (g2 if i % 3 == 1 else g).replay()
        b.run()
        if i % 7 == 6:                                  # the last tokens rejected
            undo.replay()
            b.back()
        for name in ("out", "h", "n"):
            assert (getattr(a, name) == getattr(b, name)).all()
        assert (a.out[4:] == 7.0).all() and (a.h[4:] == 7.0).all()      # the row behind the last sequence
        assert (a.step.pos == b.step.pos).all() and (a.step.place == b.step.place).all()
        assert a.tables.lens.tolist() == b.tables.lens.tolist()
    assert a.tables.lens.tolist() == [35, 70, 35] and torch.isfinite(a.out.float()).all()
    assert ec.echo_get_device_error() == 0
