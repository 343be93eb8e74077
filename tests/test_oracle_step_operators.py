"""Pins for the oracle's 4-bit codes, page tables, rotary positions and gated norms.  No GPU."""
import numpy as np
import pytest

import int4_case
from oracle import block, cache, int4, norms, rotary, tables

F32 = np.float32


def test_codes_by_hand():
    x = np.zeros(64, F32)
    x[:6] = [7, -3.5, 3.5, 0.5, 0.49, -7]          # scale 1: halves go away from zero
    x[32:35] = [15, -14, 1]                        # 15 / 7 = 2.14..: 2.25 of 5 bits (18 / 8)
    codes, scale, bad = int4.quantize(x)
    assert not bad and list(scale) == [1, 2.25]
    assert list(codes[:6]) == [7, -4, 4, 1, 0, -7] and list(codes[32:35]) == [7, -6, 0]
    word = int4.pack(codes)[:4].view("<u4")[0]
    assert [(int(word) >> s) & 15 for s in (0, 16, 4, 20, 8, 24)] == [15, 4, 12, 9, 8, 1]


def test_codes_are_as_near_as_they_can_be():
    g = np.random.default_rng(1)
    x = (g.standard_normal((50, 64)) * 10.0 ** g.integers(-30, 30, (50, 1))).astype(F32)
    x[3], x[4, :32] = 0, 1e-38
    codes, scale, _ = int4.quantize(x)
    u, s = cache.round_bf16(x).astype(np.float64), np.repeat(scale.astype(np.float64), 32, axis=1)
    assert np.abs(codes).max() == 7 and (np.abs(u - codes * s) <= s / 2).all()
    a = np.abs(u).reshape(50, 2, 32).max(axis=2)
    assert (a <= 7 * scale).all()
    assert (a > 7 * scale * 16 / 17.0001)[scale > int4.LEAST].all()      # one step of 5 bits less is too little
    m = np.frexp(scale)[0] * 32
    assert (m == np.floor(m)).all()
    v = (codes * s).astype(F32)
    assert np.array_equal(cache.round_bf16(v), v)
    assert np.array_equal(int4.unpack(int4.pack(codes)), codes)
    assert np.array_equal(int4.values(int4.pack(codes), scale), v)


@pytest.mark.parametrize("value", [np.inf, -np.inf, np.nan, 3.4e38])
def test_codes_of_what_is_not_finite(value):
    x = np.ones((2, 32), F32)
    x[1, 5] = value                                # 3.4e38 is infinite in bf16
    codes, scale, bad = int4.quantize(x)
    assert bad and not codes[1].any() and codes[0].all() and scale[0] == int4.scale_of(1.0)
    assert np.isnan(scale[1]) if np.isnan(value) else scale[1] == np.inf


def test_cases_of_four_bits():
    c = int4_case.make(16, 2, 64, [20, 0, 3], [1, 0, 3])
    v = c.values
    assert np.isfinite(v[c.table[0, 0]]).all() and v.shape == (*c.pages.shape[:4], 64)
    assert np.isfinite(v[c.table[0, 1], :, :, :4]).all() and not np.isfinite(v[c.table[0, 1], :, :, 4:]).all()


def test_tables_by_hand():
    t = tables.Tables(6, 16, 3, 4)
    lens, row0, maps = t.extend([2, 0], [17, 3], 22)
    assert t.pages == [[2], [], [0, 1]] and t.free == [5, 4, 3] and lens == [17, 3] and row0 == [0, 17, 20]
    assert maps[:2] == [(0, 0, 0), (1, 1, 0)] and maps[16:] == [(16, 16, 0), (32, 0, 1), (33, 1, 1), (34, 2, 1),
                                                                (-1, -1, -1), (-1, -1, -1)]
    lens, row0, maps = t.extend([0], [14], 14)
    assert t.pages[0] == [2, 3] and maps[12] == (47, 15, 0) and maps[13] == (48, 16, 0)
    assert t.shorten([0], [14]) and t.pages[0] == [2] and t.free == [5, 4, 3]
    assert t.shorten([2, 0], [99, 3]) and t.lens == [0, 0, 0] and t.free == [5, 4, 3, 2, 1, 0]


def test_tables_that_cannot_be_served():
    t = tables.Tables(4, 16, 3, 3)
    assert t.extend([0], [40], 40) is not None
    before = ([list(p) for p in t.pages], list(t.lens), list(t.free))
    for slots, rows, n in (([1], [17], 17), ([0], [9], 9), ([0, 0], [1, 1], 2), ([3], [1], 1), ([-1], [1], 1),
                           ([1], [-1], 4), ([1], [5], 4)):
        assert t.extend(slots, rows, n) is None
    assert not t.shorten([0, 0], [1, 1]) and not t.shorten([0], [-1]) and not t.shorten([3], [1])
    assert before == ([list(p) for p in t.pages], list(t.lens), list(t.free))


def test_tables_undo():
    g = np.random.default_rng(2)
    t = tables.Tables(200, 32, 9, 40, free=g.permutation(200))
    t.extend(list(range(9)), [int(n) for n in g.integers(0, 300, 9)], 3000)
    for _ in range(20):
        slots = [int(s) for s in g.permutation(9)[:g.integers(1, 9)]]
        rows = [int(n) for n in g.integers(0, 200, len(slots))]
        before = ([list(p) for p in t.pages], list(t.lens), list(t.free))
        if t.extend(slots, rows, 5000) is not None:
            used = [p for pages in t.pages for p in pages]
            assert sorted(used + t.free) == list(range(200))
            t.shorten(slots, rows)
        assert before == ([list(p) for p in t.pages], list(t.lens), list(t.free))


def test_turns_by_hand():
    x = np.arange(8, dtype=F32)[None]
    freq = np.array([np.pi / 2, np.pi / 4])
    y, mass = rotary.turn(x, [1], 8, [2], freq)
    r = np.sqrt(0.5)
    assert np.allclose(y[0], [-1, 0, (2 - 3) * r, (3 + 2) * r, 4, 5, 6, 7]) and list(mass[0]) == [1, 1, 5, 5, 0, 0, 0, 0]
    y, _ = rotary.turn(x, [1], 8, [2], freq, layout="halves", size=2.0)
    assert np.allclose(y[0, :4], [-4, 2 * (1 - 3) * r, 0, 2 * (3 + 1) * r])
    assert np.allclose(rotary.turn(x, [[0, 2]], 8, [1, 1], freq)[0][0], [0, 1, -3, 2, 4, 5, 6, 7])
    assert np.array_equal(rotary.turn(x, [0], 8, [2], freq)[0], x)


def test_turns_depend_on_distances():
    g = np.random.default_rng(3)
    q, k = g.standard_normal((2, 1, 32))
    freq, _ = rotary.frequencies([16], 10000.0)
    dots = [(rotary.turn(q, [a + 7], 32, [16], freq)[0] * rotary.turn(k, [a], 32, [16], freq)[0]).sum()
            for a in (0, 5, 100000)]
    assert np.allclose(dots, dots[0])
    y, _ = rotary.turn(q, [33], 32, [16], freq, size=1.5)
    back, _ = rotary.turn(y, [33], 32, [16], freq, size=1.5, inverse=True)
    assert np.allclose(back, 2.25 * q)                     # the transposed map, sizes and all


def test_slower_turns():
    plain, _ = rotary.frequencies([64], 10000.0)
    assert np.allclose(rotary.frequencies([64], 10000.0, "linear", 4.0)[0] * 4, plain)
    ntk, _ = rotary.frequencies([64], 10000.0, "ntk", 4.0)
    assert ntk[0] == 1 and np.isclose(ntk[-1] * 4, plain[-1])
    yarn, size = rotary.frequencies([64], 10000.0, "yarn", 4.0, 4096)
    turns = 4096 * plain / (2 * np.pi)
    assert np.allclose(yarn[turns >= 32], plain[turns >= 32]) and np.allclose(yarn[turns <= 1] * 4, plain[turns <= 1])
    assert (np.diff(yarn) < 0).all() and np.isclose(size, 0.1 * np.log(4) + 1)


def test_norms_by_hand():
    x, y = np.array([[1.0, 3.0]]), np.array([[3.0, 4.0]])
    h, n = norms.gated(x, y, gate=[[2.0, 0.5]], scale=[[1.0, 0.0]], shift=[[0.0, 10.0]], after="rms", eps=0.0, beta=0.5)
    r = np.sqrt(12.5)
    assert np.allclose(h, [[1 + 3 / r, 3 + 0.25 * 4 / r]])
    assert np.allclose(n, [[-2.0, 11.0]])
    g = np.random.default_rng(4)
    x = g.standard_normal((5, 64))
    assert np.allclose(norms.gated(x)[1], block.layer_norm(x))
    assert np.array_equal(norms.gated(x, x, gate=0 * x)[0], x)
    n = norms.norm(x, "layer", eps=0.0)
    assert np.allclose(n.mean(axis=1), 0) and np.allclose(n.var(axis=1), 1)
