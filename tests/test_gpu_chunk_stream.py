"""Blocks run chunk by chunk over paged keys and values (pipeline.ChunkStream) against the
oracle's block with a frame-causal mask over the whole clip, in fp64.

Tolerances: those of the block step (max 2e-2 normwise per token, mean 5e-3), on bf16
pages.  int8 pages add a quantisation error of up to half a code in 127 of a head's largest
key or value: the oracle quantises its own keys and values by the same rule, and the same
bars hold against it.
"""
import numpy as np
import pytest

pytestmark = pytest.mark.gpu

import oracle                                      # noqa: E402
from synth import TINY_256, generate as G          # noqa: E402

F32 = np.float32
W = TINY_256


@pytest.fixture(scope="module")
def ec():
    import torch
    if not torch.cuda.is_available():
        pytest.skip("needs a GPU")
    from paper_2608_02474_gb300 import echocache
    return echocache


def attention(Q, K, V, H, tops, int8):
    """Row i over the first tops[i] keys."""
    d = Q.shape[1] // H
    if int8:
        deq = lambda x: np.concatenate([                       # noqa: E731
            (lambda q, s, _: q.astype(np.float64) * s[:, None])(*oracle.cache.quantize_rows(
                oracle.cache.round_bf16(x[:, h * d:h * d + d].astype(F32)))) for h in range(H)], axis=1)
        K, V = deq(K), deq(V)
    out = np.zeros_like(Q)
    for i, n in enumerate(tops):
        out[i] = oracle.block.mha(Q[i:i + 1], K[:n], V[:n], H)[0]
    return out


def reference(x, weights, conds, frame, int8):
    B = oracle.block
    n = x.shape[0]
    tops = [min(n, (p // frame + 1) * frame) for p in range(n)]
    for w, cond in zip(weights, conds):
        x = x.astype(np.float64)
        n1 = B.layer_norm(x)
        lin = lambda a, m: B.linear(a, w["W" + m], w["b" + m])     # noqa: E731
        h1 = x + lin(attention(lin(n1, "q"), lin(n1, "k"), lin(n1, "v"), W.H, tops, int8), "o")
        kc, vc = B.cross_kv(cond, w)
        h2 = h1 + lin(attention(lin(B.layer_norm(h1), "qc"), kc, vc, W.H, [len(cond)] * n, int8), "oc")
        x = h2 + B.linear(B.gelu_tanh(B.linear(B.layer_norm(h2), w["W1"], w["b1"])), w["W2"], w["b2"])
        x = oracle.cache.round_bf16(x.astype(F32))
    return x


@pytest.mark.parametrize("int8", [False, True])
@pytest.mark.parametrize("frame", [1, 24])
def test_chunks_of_several_clips(ec, int8, frame):
    """Three clips, chunks of other lengths in each step, one clip closed and its pages taken
    by the next."""
    import torch
    from paper_2608_02474_gb300.pipeline import ChunkStream
    weights = [G.block_weights(W, l) for l in range(2)]
    conds = {c: [G.random_rows(n, W.D, seed=40 + c) for _ in weights] for c, n in ((0, 32), (1, 7), (2, 90))}
    total = {0: 5 * 24, 1: 3 * 24, 2: 4 * 24}
    xs = {c: G.random_rows(n, W.D, seed=50 + c) for c, n in total.items()}
    blocks = [ec.DeviceBlock.from_host(w, np.zeros((1, W.D), F32)) for w in weights]
    bf = lambda a: torch.from_numpy(np.ascontiguousarray(a)).to("cuda", torch.bfloat16)   # noqa: E731

    def cond_kv(c):
        return [ec.echo_precompute_cross_kv(bf(conds[c][l]), torch.cat([bf(w["Wkc"]), bf(w["Wvc"])]),
                                            torch.cat([bf(w["bkc"]), bf(w["bvc"])]))
                for l, w in enumerate(weights)]

    # room for clips 0 and 1, not for a third: 120 and 72 tokens in pages of 16 are 13
    st = ChunkStream(blocks, W.H, W.d, frame, n_pages=14, cond_pages=8, page_tokens=16,
                     kind=ec.CACHE_INT8 if int8 else ec.CACHE_BF16)
    got = {c: [] for c in total}
    at = dict.fromkeys(total, 0)

    def step(lengths):
        y = st.step({c: bf(xs[c][at[c]:at[c] + n]) for c, n in lengths.items()})
        for c, n in lengths.items():
            assert y[c].shape == (n, W.D)
            got[c].append(y[c].float().cpu().numpy())
            at[c] += n

    with pytest.raises(ValueError, match="not open"):
        st.step({0: bf(xs[0][:1])})
    st.open(0, cond_kv(0))
    st.open(1, cond_kv(1))
    with pytest.raises(MemoryError):
        st.open(2, cond_kv(2))
    chunk = 24 if frame > 1 else 17
    step({0: chunk, 1: chunk})
    step({0: chunk})
    step({1: 72 - at[1], 0: chunk})                    # several frames at once, other order
    with pytest.raises(MemoryError):
        st.step({0: bf(np.zeros((140, W.D), F32)), 1: bf(np.zeros((140, W.D), F32))})
    st.close(1)
    st.open(2, cond_kv(2)[:2])
    step({2: chunk, 0: 120 - at[0]})
    st.close(0)
    if frame == 1:
        step({2: 1})                                   # single tokens
        step({2: 1})
    step({2: 96 - at[2]})
    st.close(2)
    assert sorted(st.self_table.free) == list(range(14)) and sorted(st.cond_table.free) == list(range(8))
    assert ec.echo_get_device_error() == 0
    for c in total:
        y = np.concatenate(got[c])
        ref = reference(G.to_bf16_values(xs[c]), weights, [G.to_bf16_values(a) for a in conds[c]], frame, int8)
        rel = np.abs(y - ref).max(axis=1) / np.abs(ref).max(axis=1)
        mean = np.abs(y - ref).sum() / np.abs(ref).sum()
        assert rel.max() <= 2e-2 and mean <= 5e-3, (c, rel.max(), mean)


@pytest.mark.parametrize("int8", [False, True])
def test_a_frame_that_comes_in_parts(ec, int8):
    """Tokens see their frame as far as it has come.  One block, whose keys and values do not
    depend on what earlier tokens saw: each chunk's rows are those of the clip up to it."""
    import torch
    from paper_2608_02474_gb300.pipeline import ChunkStream
    w = G.block_weights(W, 0)
    cond, x = G.random_rows(19, W.D, seed=61), G.random_rows(90, W.D, seed=62)
    bf = lambda a: torch.from_numpy(np.ascontiguousarray(a)).to("cuda", torch.bfloat16)   # noqa: E731
    kv = ec.echo_precompute_cross_kv(bf(cond), torch.cat([bf(w["Wkc"]), bf(w["Wvc"])]),
                                     torch.cat([bf(w["bkc"]), bf(w["bvc"])]))
    st = ChunkStream([ec.DeviceBlock.from_host(w, np.zeros((1, W.D), F32))], W.H, W.d, 24, n_pages=6, cond_pages=2,
                     page_tokens=16, kind=ec.CACHE_INT8 if int8 else ec.CACHE_BF16)
    st.open(0, [kv])
    lo = 0
    for n in (17, 1, 30, 24, 18):                      # up to 17, 18, 48, 72, 90 of frames of 24
        y = st.step({0: bf(x[lo:lo + n])})[0].float().cpu().numpy()
        lo += n
        ref = reference(G.to_bf16_values(x[:lo]), [w], [G.to_bf16_values(cond)], 24, int8)[-n:]
        rel = np.abs(y - ref).max(axis=1) / np.abs(ref).max(axis=1)
        assert rel.max() <= 2e-2 and np.abs(y - ref).sum() / np.abs(ref).sum() <= 5e-3, (lo, rel.max())
    assert ec.echo_get_device_error() == 0
