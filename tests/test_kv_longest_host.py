"""The longest sequence of a batch, as the host tells the library: what is refused, and what the page
tables on the device tell.  No GPU."""
import ctypes
import os
import types

from test_device_tables_host import calls, pipeline, stream   # noqa: F401
from test_kv_abi import BATCH, POOL, ec                       # noqa: F401


def test_bad_numbers(ec):                                     # noqa: F811
    p, b = (ctypes.byref(s) for s in (ec.KVPoolC(**POOL), ec.KVBatchC(**BATCH, max_len=-1)))
    L, x = ec.lib(), POOL["pages"]
    assert (L.echo_kv_write(p, b, x, x, 128, 0, None), L.echo_kv_read(p, b, x, x, 128, 0, None),
            L.echo_kv_attention(p, b, x, 128, 2, 0, x, 128, x, 1 << 40, None)) == (2, 2, 2)
    assert L.echo_kv_attention_workspace_size(p, b, 2) == 0
    # the workspace does not go by it
    sizes = {n: L.echo_kv_attention_workspace_size(p, ctypes.byref(ec.KVBatchC(**BATCH, max_len=n)), 2)
             for n in (0, 1, 48, 10 ** 6)}
    assert len(set(sizes.values())) == 1 and sizes[0] > 0


def test_the_struct_is_the_headers(ec):                       # noqa: F811
    """Its fields after max_rows, where callers without it have left zeros."""
    root = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
    head = open(os.path.join(root, "include", "echocache.h")).read()
    fields = head[:head.index("} echo_kv_batch;")].rsplit("typedef struct {", 1)[1]
    assert fields.index("max_rows;") < fields.index("max_len;")
    assert ec.KVBatchC.max_len.offset == ec.KVBatchC.max_rows.offset + 4
    assert ec.KVBatchC(**BATCH).max_len == 0


def test_what_the_tables_on_the_device_tell(calls):           # noqa: F811
    t = pipeline.DevicePageTable(100, 16, 3, "cpu")
    for c in "abc":
        t.open(c)
    assert t.extend({"a": 40, "b": 700}).batch.max_len == 700
    assert t.extend({"a": 1, "c": 0}).batch.max_len == 41
    assert t.extend({"c": 0}).batch.max_len == 0
    assert t.extend({}).batch.max_len == 0


def test_a_step_hands_both_on(calls, monkeypatch):            # noqa: F811
    import torch
    made = []
    monkeypatch.setattr(pipeline.ec, "KVBatch", lambda *a: made.append(a) or types.SimpleNamespace())
    st = stream()
    st.open(0, [torch.zeros(20, 256, dtype=torch.bfloat16) for _ in range(2)])
    st.step({0: torch.zeros(18, 128, dtype=torch.bfloat16)})
    assert [a[-1] for a in made] == [20]
    assert st.self_table.lens[0] == 18
