"""What the host keeps of page tables on the GPU, and ChunkStream on them where a call is refused
or fails.  The library's calls are stand-ins that compute nothing.  No GPU."""
import types

import pytest
import torch

from paper_2608_02474_gb300 import pipeline

D, H = 128, 2


class Tables:
    @staticmethod
    def empty(n_pages, page_tokens, n_slots, max_pages, device):
        return types.SimpleNamespace(max_pages=max_pages)


class Step:
    @staticmethod
    def empty(tables, n_seqs, n_rows, max_rows=None):
        batch = types.SimpleNamespace(table=None, lens=None, row0=None, max_rows=max_rows)
        return types.SimpleNamespace(n_seqs=n_seqs, n_rows=n_rows, batch=batch, place=object(), pos=object(), seq=object())


class Block:
    tensors = {k: None for k in ("Wkv", "bkv", "Wq", "bq", "Wo", "bo", "Wqc", "bqc", "Woc", "boc", "W1", "b1", "W2",
                                 "b2")}


@pytest.fixture
def calls(monkeypatch):
    """The library's calls by name; the n-th from now on raises where calls.fail = n."""
    ec, made = pipeline.ec, types.SimpleNamespace(names=[], fail=None)

    def call(name):
        def f(*args, **kw):
            if made.fail is not None:
                made.fail -= 1
                if made.fail < 0:
                    made.fail = None
                    raise RuntimeError("a call failed")
            made.names.append(name)
            if name == "echo_gated_norm":
                return torch.zeros(args[1].shape), torch.zeros(args[1].shape)
            return torch.zeros(args[0].shape[0], 2 * D) if name == "echo_linear" else torch.zeros(1)
        return f

    for name in ("echo_kv_extend", "echo_kv_shorten", "echo_gated_norm", "echo_linear", "echo_kv_write_at",
                 "echo_kv_attention", "echo_rotary"):
        monkeypatch.setattr(ec, name, call(name))
    monkeypatch.setattr(ec, "echo_kv_attention", lambda pool, batch, q, **kw: call("echo_kv_attention")(pool) is None or q)
    monkeypatch.setattr(ec, "KVTables", Tables)
    monkeypatch.setattr(ec, "KVStep", Step)
    monkeypatch.setattr(ec, "KVBatch", lambda *a: object())
    monkeypatch.setattr(ec, "KVPool", types.SimpleNamespace(empty=lambda *a: object()))
    monkeypatch.setattr(pipeline.DevicePageTable, "_numbers", lambda self, rows: ([self.slots[c] for c in rows], list(rows.values())))
    return made


def test_counts_of_pages_and_slots(calls):
    t = pipeline.DevicePageTable(10, 16, 2, "cpu")
    t.open("a")
    t.open("b")
    with pytest.raises(MemoryError):
        t.open("c")
    with pytest.raises(ValueError):
        t.open("a")
    assert t.slots == {"a": 0, "b": 1}
    t.extend({"a": 17, "b": 1})
    assert t.n_free == 7 and t.lens == {"a": 17, "b": 1}
    with pytest.raises(MemoryError):
        t.extend({"a": 100, "b": 40})
    assert t.n_free == 7 and t.lens == {"a": 17, "b": 1}
    t.shorten({"a": 1})
    assert t.n_free == 8 and t.lens["a"] == 16
    t.close("a")
    assert t.n_free == 9 and t.free_slots == [0]
    t.open("c")
    assert t.slots["c"] == 0 and calls.names.count("echo_kv_shorten") == 2


def test_counts_that_the_tables_would_not_follow(calls):
    """More than a clip has: all of it, as on the device; negative numbers are refused before any call."""
    t = pipeline.DevicePageTable(10, 16, 2, "cpu")
    t.open("a")
    t.extend({"a": 40})
    made = len(calls.names)
    for f in (t.extend, t.shorten):
        with pytest.raises(ValueError):
            f({"a": -1})
    assert len(calls.names) == made and t.lens == {"a": 40} and t.n_free == 7
    t.shorten({"a": 41})
    assert t.lens == {"a": 0} and t.n_free == 10


def stream(**kw):
    return pipeline.ChunkStream([Block(), Block()], H, D // H, 4, n_pages=6, cond_pages=3, page_tokens=16, device="cpu",
                                device_tables=True, **kw)


def cond(n):
    return [torch.zeros(n, 2 * D, dtype=torch.bfloat16) for _ in range(2)]


def state(st):
    return [(dict(t.lens), dict(t.slots), t.n_free, sorted(t.free_slots)) for t in (st.self_table, st.cond_table)]


def test_a_step_that_fails_is_taken_back(calls):
    st = stream()
    st.open(0, cond(20))
    x = torch.zeros(18, D, dtype=torch.bfloat16)
    before = state(st)
    calls.names.clear()
    st.step({0: x})
    n = len(calls.names)
    assert n > 20 and state(st) != before
    st.self_table.shorten({0: 18})
    assert state(st) == before
    for i in range(1, n):                      # the first call is the extension itself
        calls.fail = i
        with pytest.raises(RuntimeError):
            st.step({0: x})
        assert state(st) == before, i
    calls.fail = 0
    with pytest.raises(RuntimeError):
        st.step({0: x})
    assert state(st) == before


def test_opening_undoes_itself(calls):
    st = stream(max_clips=1)
    for fail in (0, 1, 2):
        calls.fail = fail
        before = state(st)
        with pytest.raises(RuntimeError):
            st.open(0, cond(20))
        calls.fail = None
        assert state(st) == before
    with pytest.raises(MemoryError):
        st.open(0, cond(50))
    assert state(st) == before
    st.open(0, cond(20))
    with pytest.raises(MemoryError):
        st.open(1, cond(1))
    st.close(0)
    assert state(st) == before
