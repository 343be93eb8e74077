"""Pins for the oracle's paged key/value cache.  No GPU."""
import numpy as np
import pytest

import kv_case
from oracle import cache as C
from oracle import paged as P

F32 = np.float32


def test_hand_worked_write_and_read():
    """Two pages of 16 in reverse order, one head of 64: positions 15 and 16 fall on the
    last slot of page 1 and the first of page 0."""
    pages, scale = np.zeros((2, 2, 1, 16, 64), np.int8), np.zeros((2, 2, 1, 16), F32)
    table = np.array([[1, 0]], np.int32)
    k = np.zeros((2, 64), F32)
    k[0, :3], k[1, 0] = [127, -63.5, 0.5], 254
    P.write(pages, scale, table, [17], [0, 2], k, -k)
    assert list(pages[1, 0, 0, 15, :3]) == [127, -64, 0] and scale[1, 0, 0, 15] == 1
    assert pages[0, 0, 0, 0, 0] == 127 and scale[0, 0, 0, 0] == 2
    assert list(pages[1, 1, 0, 15, :3]) == [-127, 64, 0]
    assert not pages[0, :, :, 1:].any() and not pages[1, :, :, :15].any()
    rk, rv = P.read(pages, scale, table, [17], [0, 2], 2)
    assert list(rk[0, :3]) == [127, -64, 0] and rk[1, 0] == 254 and rv[1, 0] == -254


@pytest.mark.parametrize("form", ["bf16", "int8"])
def test_write_then_read(form):
    c = kv_case.make(form, 16, 3, 64, [40, 0, 17], [40, 0, 5])
    g = np.random.default_rng(1)
    k, v = (g.standard_normal((45, 192)).astype(F32) for _ in range(2))
    P.write(c.pages, c.scale, c.table, c.lens, c.row0, k, v)
    for got, x in zip(P.read(c.pages, c.scale, c.table, c.lens, c.row0, 45), (k, v)):
        if form == "bf16":
            assert np.array_equal(got, C.round_bf16(x))
        else:
            a = np.abs(x.reshape(45, 3, 64)).max(2)[..., None] / 127
            assert (np.abs(got - x).reshape(45, 3, 64) <= a * (0.5 + 2.0 ** -14)).all()


def test_rows_before_the_start_are_left_out():
    c = kv_case.make("bf16", 16, 1, 64, [3], [5])
    k = np.ones((5, 64), F32) * np.arange(5, dtype=F32)[:, None]
    P.write(c.pages, None, c.table, c.lens, c.row0, k, k)
    got, _ = P.read(c.pages, None, c.table, c.lens, c.row0, 5)
    assert list(got[:, 0]) == [0, 0, 2, 3, 4]


@pytest.mark.parametrize("form", ["bf16", "int8"])
@pytest.mark.parametrize("group", [1, 3])
def test_attention_is_the_dense_softmax(form, group):
    c = kv_case.make(form, 32, 2, 64, [70, 33], [4, 33])
    Hq = 2 * group
    q = kv_case.queries(37, Hq * 64, 3)
    out, mass = P.attend(c.pages, c.scale, c.table, c.lens, c.row0, q, Hq)
    for b, (lo, hi) in enumerate(((0, 4), (4, 37))):
        k, v = P.keys_values(c.pages, c.scale, c.table, int(c.lens[b]), b)
        for h in range(Hq):
            s = q[lo:hi, h * 64:h * 64 + 64].astype(np.float64) @ k[:, h // group].T / 8
            p = np.exp(s)
            p /= p.sum(1, keepdims=True)
            assert np.allclose(out[lo:hi, h * 64:h * 64 + 64], p @ v[:, h // group], atol=1e-12)
    assert (mass >= np.abs(out) - 1e-12).all()


def test_page_order_changes_nothing():
    c = kv_case.make("int8", 16, 1, 64, [50], [2], spare=0)
    q = kv_case.queries(2, 64, 5)
    a, _ = P.attend(c.pages, c.scale, c.table, c.lens, c.row0, q, 1)
    perm = np.array([2, 0, 3, 1])
    inv = np.argsort(perm)
    b, _ = P.attend(c.pages[perm], c.scale[perm], inv[c.table], c.lens, c.row0, q, 1)
    assert np.array_equal(a, b)


@pytest.mark.parametrize("cb", [1, 7, 16, 100])
def test_causal_rows_see_a_shorter_sequence(cb):
    c = kv_case.make("bf16", 16, 1, 64, [45], [45])
    q = kv_case.queries(45, 64, 6)
    out, _ = P.attend(c.pages, None, c.table, c.lens, c.row0, q, 1, cb)
    for p in (0, 6, 7, 20, 44):
        top = min(45, (p // cb + 1) * cb)
        one, _ = P.attend(c.pages, None, c.table, [top], [0, 1], q[p:p + 1], 1)
        assert np.allclose(out[p], one[0], atol=1e-13)


def test_no_key_no_output():
    c = kv_case.make("bf16", 16, 1, 64, [0, 2], [3, 4])
    q = kv_case.queries(7, 64, 7)
    out, _ = P.attend(c.pages, None, c.table, c.lens, c.row0, q, 1, 1)
    assert not out[:5].any() and out[5:].all()      # the first two of four rows stand before 0
