"""ChunkStream's bookkeeping where a call is refused or fails: the clips stay as they were.
The library's calls are stand-ins that compute nothing.  No GPU."""
import pytest
import torch

from paper_2608_02474_gb300 import pipeline

D, H = 128, 2


class Pool:
    @staticmethod
    def empty(*args):
        return object()


class Block:
    tensors = {k: None for k in ("Wkv", "bkv", "Wq", "bq", "Wo", "bo", "Wqc", "bqc", "Woc", "boc", "W1", "b1",
                                 "W2", "b2")}


@pytest.fixture
def stream(monkeypatch):
    """A stream of two blocks, whose n-th next library call raises where st.fail = n."""
    ec, calls = pipeline.ec, []

    def call(*args, **kw):
        calls.append(args)
        if st.fail is not None and len(calls) > st.fail:
            raise RuntimeError("a call failed")
        return args[0] if isinstance(args[0], torch.Tensor) else torch.zeros(len(args[2]), D)

    for name in ("echo_layernorm", "echo_linear", "echo_kv_write", "echo_kv_attention"):
        monkeypatch.setattr(ec, name, call)
    monkeypatch.setattr(ec, "KVPool", Pool)
    monkeypatch.setattr(pipeline.PageTable, "batch", lambda self, rows, device: call([], rows, range(sum(rows.values()))))
    st = pipeline.ChunkStream([Block(), Block()], H, D // H, 4, n_pages=6, cond_pages=3, page_tokens=16, device="cpu")
    st.calls, st.fail = calls, None
    return st


def cond(n, layers=2):
    return [torch.zeros(n, 2 * D, dtype=torch.bfloat16) for _ in range(layers)]


def rows(n, cols=D, dtype=torch.bfloat16):
    return torch.zeros(n, cols, dtype=dtype)


def state(st):
    return [(dict(t.lens), {c: list(p) for c, p in t.pages.items()}, sorted(t.free))
            for t in (st.self_table, st.cond_table)]


def steps_after(st, fail, call):
    st.calls.clear()
    st.fail = fail
    with pytest.raises(RuntimeError):
        call()
    st.fail = None


def test_a_step_that_fails_takes_its_tokens_back(stream):
    st = stream
    st.open(0, cond(5))
    st.open(1, cond(20))
    st.step({0: rows(15), 1: rows(3)})
    before = state(st)
    for fail in (0, 1, 3, 4, 6, 20):
        steps_after(st, fail, lambda: st.step({1: rows(20), 0: rows(2)}))
        assert state(st) == before, fail
    st.step({1: rows(20), 0: rows(2)})
    assert st.self_table.lens == {0: 17, 1: 23} and [len(p) for p in st.self_table.pages.values()] == [2, 2]


def test_chunks_are_looked_at_before_anything_is_taken(stream):
    st = stream
    st.open(0, cond(5))
    before = state(st)
    for bad, error in ((rows(2, D - 8), ValueError), (rows(2, D + 8), ValueError), (rows(2)[0], ValueError),
                       (rows(2, dtype=torch.float16), TypeError), (rows(2, dtype=torch.int32), TypeError)):
        st.calls.clear()
        with pytest.raises(error):
            st.step({0: bad})
        assert state(st) == before and not st.calls
    with pytest.raises(MemoryError):
        st.step({0: rows(97)})
    assert state(st) == before


def test_a_chunk_of_a_wider_tensor_is_made_contiguous(stream):
    stream.open(0, cond(1))
    stream.calls.clear()
    stream.step({0: rows(4, 2 * D)[:, D:]})
    x = [a[0] for a in stream.calls if isinstance(a[0], torch.Tensor)][0]
    assert x.shape == (4, D) and x.is_contiguous()


def test_no_chunks_and_chunks_of_no_rows(stream):
    stream.open(0, cond(1))
    assert stream.step({}) == {}
    y = stream.step({0: rows(0, dtype=torch.float32)})
    assert y[0].shape == (0, D) and y[0].dtype == torch.bfloat16 and stream.self_table.lens == {0: 0}


def test_opening_looks_at_every_layer(stream):
    st = stream
    st.open(7, cond(5))
    before = state(st)
    for bad in (cond(5, 1), cond(5, 3), [], [cond(5, 1)[0], cond(6, 1)[0]], [cond(5, 1)[0], rows(5)]):
        st.calls.clear()
        with pytest.raises(ValueError):
            st.open(1, bad)
        assert state(st) == before and not st.calls
    with pytest.raises(MemoryError):
        st.open(1, cond(33))
    with pytest.raises(ValueError):
        st.open(7, cond(5))
    assert state(st) == before


def test_an_opening_that_fails_leaves_the_clip_closed(stream):
    st = stream
    before = state(st)
    for fail in (0, 1, 2):
        steps_after(st, fail, lambda: st.open(1, cond(20)))
        assert state(st) == before, fail
    st.open(1, cond(20))
    assert st.cond_table.lens == {1: 20} and st.self_table.lens == {1: 0}


def test_pages_are_given_back_by_the_tokens_that_needed_them():
    t = pipeline.PageTable(6, 16)
    t.open(1)
    t.open(2)
    t.extend({1: 40, 2: 16})
    t.shorten({1: 8})                                 # 32 of 40: the third page
    assert t.lens == {1: 32, 2: 16} and len(t.pages[1]) == 2 and len(t.free) == 3
    t.shorten({1: 1, 2: 16})
    assert t.lens == {1: 31, 2: 0} and len(t.pages[1]) == 2 and t.pages[2] == []
    t.extend({2: 64})
    assert sorted(t.pages[1] + t.pages[2]) == list(range(6))
