"""Rotary positions against the oracle in fp64.

Tolerance.  An angle is p f modulo one turn: the fraction of a turn is held to 2^-32 and
its fp32 number of half turns to 2^-25, together below 2^-23 radians; sine and cosine come
with up to 2 units of 2^-24, their product with `size`, the two products and the sum with one
rounding each: below 2^-21 size (|x1| + |x2|) in all.  f itself is an fp64 power, off by up
to 2^-51 of itself: below 2^-30 radians at 2^20 positions.  The result is rounded once, by up
to 2^-8 (bf16) or 2^-24 (fp32) of itself.
"""
import numpy as np
import pytest

pytestmark = pytest.mark.gpu

from oracle import rotary as R                     # noqa: E402

F32 = np.float32


@pytest.fixture(scope="module")
def ec():
    import torch
    if not torch.cuda.is_available():
        pytest.skip("needs a GPU")
    from paper_2608_02474_gb300 import echocache
    return echocache


def tensor(n, heads, d, t, seed):
    import torch
    x = torch.from_numpy(np.random.default_rng(seed).standard_normal((n, heads * d)).astype(F32)).cuda()
    return x.to(torch.bfloat16) if t == "bf16" else x


def host(t):
    return t.float().cpu().numpy()


def i32(a):
    import torch
    return torch.from_numpy(np.ascontiguousarray(a).astype(np.int32)).cuda()


def check(got, x, pos, d, axis_pairs, freq, size, layout, inverse=False, frame=None):
    want, mass = R.turn(host(x), pos, d, axis_pairs, freq, size, layout, inverse, frame)
    rounding = 2.0 ** -8 if got.element_size() == 2 else 2.0 ** -24
    off = np.abs(host(got) - want) - (rounding * np.abs(want) + 2.0 ** -21 * mass)
    assert off.max(initial=-1) <= 0, float(off.max())
    n = sum(axis_pairs)
    a, b = host(got).reshape(len(want), -1, d), host(x).reshape(len(want), -1, d)
    assert np.array_equal(a[:, :, 2 * n:], b[:, :, 2 * n:])              # as they were


SHAPES = [
    # d, pairs: whole heads, parts, odd parts
    (128, 64), (64, 32), (128, 32), (128, 20), (64, 10), (64, 7), (128, 1), (128, 63), (8, 3), (256, 128), (24, 12),
    (80, 21), (256, 1),
]
LAYOUT = pytest.mark.parametrize("layout", ["pairs", "halves"])
TYPES = pytest.mark.parametrize("t", ["bf16", "f32"])


@LAYOUT
@TYPES
@pytest.mark.parametrize("d,pairs", SHAPES)
def test_heads_and_parts(ec, d, pairs, layout, t):
    for n, Hq, H in ((1, 1, 1), (5, 3, 2), (67, 9, 1)):
        q, k = tensor(n, Hq, d, t, n), tensor(n, H, d, t, n + 1)
        pos = np.random.default_rng(n).integers(0, 2 ** 20, n)
        pos[0] = 0
        plan = ec.Rotary(d, pairs, layout=layout)
        freq, size = R.frequencies([pairs], 10000.0)
        for inverse in (False, True):
            a, b = ec.echo_rotary(plan, i32(pos), q, k, inverse=inverse)
            check(a, q, pos, d, [pairs], freq, size, layout, inverse)
            check(b, k, pos, d, [pairs], freq, size, layout, inverse)
            c = ec.echo_rotary(plan, i32(pos), q, inverse=inverse)
            assert (c == a).all()
        # in place, both or one
        q2, k2 = q.clone(), k.clone()
        ec.echo_rotary(plan, i32(pos), q2, k2, q_out=q2, k_out=k2)
        a, b = ec.echo_rotary(plan, i32(pos), q, k)
        assert (q2 == a).all() and (k2 == b).all()
        q2 = q.clone()
        _, b2 = ec.echo_rotary(plan, i32(pos), q2, k, q_out=q2)
        assert (q2 == a).all() and (b2 == b).all()
    assert ec.echo_get_device_error() == 0


@pytest.mark.parametrize("scaling,factor", [("none", 1.0), ("linear", 2.5), ("ntk", 8.0), ("yarn", 4.0), ("yarn", 1.0)])
@pytest.mark.parametrize("theta", [10000.0, 1e6])
def test_scaled_contexts(ec, scaling, factor, theta):
    q = tensor(33, 4, 128, "f32", 1)
    pos = np.concatenate([[0, 1, 2 ** 31 - 1, 2 ** 24 + 1], np.random.default_rng(2).integers(0, 2 ** 20, 29)])
    plan = ec.Rotary(128, 64, layout="halves", theta=theta, scaling=scaling, factor=factor, original=4096)
    freq, size = R.frequencies([64], theta, scaling, factor, 4096)
    near = pos < 2 ** 21                       # further on, fp64 frequencies are not enough for the bound above
    got = ec.echo_rotary(plan, i32(pos), q)
    check(got[near.nonzero()[0]], q[near.nonzero()[0]], pos[near], 128, [64], freq, size, "halves")
    # 2^31 positions: 2^-51 2^31 radians more at most
    want, mass = R.turn(host(q), pos, 128, [64], freq, size, "halves")
    assert (np.abs(host(got) - want) <= 2.0 ** -24 * np.abs(want) + (2.0 ** -21 + 2.0 ** -20) * mass).all()


@LAYOUT
@TYPES
@pytest.mark.parametrize("axis_pairs", [[22, 21, 21], [8, 0, 4], [1, 1, 1]])
def test_frames_rows_and_columns(ec, axis_pairs, layout, t):
    """By token index, and the same by three positions a row."""
    n = 300
    q, k = tensor(n, 2, 128, t, 3), tensor(n, 5, 128, t, 4)
    freq, size = R.frequencies(axis_pairs, 10000.0)
    pos = np.arange(n) + 5000
    plan = ec.Rotary(128, axis_pairs, layout=layout, frame=(60, 12))
    a, b = ec.echo_rotary(plan, i32(pos), q, k)
    check(a, q, pos, 128, axis_pairs, freq, size, layout, frame=(60, 12))
    check(b, k, pos, 128, axis_pairs, freq, size, layout, frame=(60, 12))
    three = np.stack([pos // 60, pos % 60 // 12, pos % 12], axis=1)
    a2, b2 = ec.echo_rotary(ec.Rotary(128, axis_pairs, layout=layout), i32(three), q, k)
    assert (a == a2).all() and (b == b2).all()


@TYPES
def test_four_axes_strides_and_rows_of_none(ec, t):
    """Columns of a wider tensor; rows of negative positions left as they were."""
    import torch
    n, d, axes = 50, 64, [5, 3, 0, 9]
    wide = tensor(n, 12, d, t, 5)
    q, k = wide[:, :4 * d], wide[:, 5 * d:7 * d]
    pos = np.random.default_rng(6).integers(0, 500, (n, 4))
    pos[7, 3], pos[20], pos[49, 0] = -1, -5, -2 ** 31
    out = torch.full((n, 5 * d), 3.0, dtype=wide.dtype, device="cuda")
    plan = ec.Rotary(d, axes)
    before = wide.clone()
    a, _ = ec.echo_rotary(plan, i32(pos), q, k, q_out=out[:, d:], k_out=k)
    live = (pos >= 0).all(axis=1).nonzero()[0]
    none = (pos < 0).any(axis=1).nonzero()[0]
    freq, size = R.frequencies(axes, 10000.0)
    check(a[live], before[:, :4 * d][live], pos[live], d, axes, freq, size, "pairs")
    check(k[live], before[:, 5 * d:7 * d][live], pos[live], d, axes, freq, size, "pairs")
    assert (out[:, :d] == 3.0).all() and (out[none] == 3.0).all() and (wide[none] == before[none]).all()
    assert (wide[:, :5 * d] == before[:, :5 * d]).all() and (wide[:, 7 * d:] == before[:, 7 * d:]).all()


def test_turned_back(ec):
    """The inverse is the transposed map: <R x, y> = <x, R' y>, and R' R is size squared; against
    differences, too (the map is linear)."""
    import torch
    n, d = 40, 128
    plan = ec.Rotary(d, 50, layout="halves", scaling="yarn", factor=8.0, original=2048)
    pos = i32(np.arange(n) * 977)
    x, y, e = (tensor(n, 3, d, "f32", s) for s in (1, 2, 3))
    fx, gy = ec.echo_rotary(plan, pos, x), ec.echo_rotary(plan, pos, y, inverse=True)
    a, b = (fx.double() * y.double()).sum(), (x.double() * gy.double()).sum()
    assert abs(a - b) <= 2.0 ** -20 * (fx.double().abs() * y.double().abs()).sum() * 2
    back = ec.echo_rotary(plan, pos, fx, inverse=True).view(n, 3, d)
    want = torch.cat([x.view(n, 3, d)[..., :100].double() * plan.size ** 2, x.view(n, 3, d)[..., 100:].double()], dim=2)
    # each turn is off by 2^-21 size (|x1| + |x2|), and |x1| + |x2| grows by sqrt 2 at most
    assert ((back - want).abs() <= 2.0 ** -19 * 2 * plan.size ** 2 * x.abs().max()).all()
    h = 2.0 ** -3
    slope = ((ec.echo_rotary(plan, pos, x + h * e).double() - ec.echo_rotary(plan, pos, x - h * e).double()) / (2 * h)
             * y.double()).sum()
    assert abs(slope - (e.double() * gy.double()).sum()) <= 2.0 ** -16 * (gy.double().abs() * e.double().abs()).sum()


def test_large_and_late(ec):
    """More rows than one walk of the grid, and a tensor beyond 2^31 values."""
    import torch
    n, H, d = 270000, 64, 128
    x = torch.empty(n, H * d, dtype=torch.bfloat16, device="cuda")
    x.normal_(generator=torch.Generator("cuda").manual_seed(1))
    pos = torch.arange(n, dtype=torch.int32, device="cuda")
    got = ec.echo_rotary(ec.Rotary(d, 64), pos, x)
    freq, size = R.frequencies([64], 10000.0)
    for at in (0, 131071, 262143, 262144, n - 1):
        check(got[at:at + 1], x[at:at + 1], np.array([at]), d, [64], freq, size, "pairs")
    assert ec.echo_get_device_error() == 0


def test_captured_stream_and_no_rows(ec):
    import torch
    q, k = tensor(9, 4, 64, "bf16", 1), tensor(9, 2, 64, "bf16", 2)
    pos, plan = i32(np.arange(9)), ec.Rotary(64, 32)
    a, b = ec.echo_rotary(plan, pos, q, k)
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    a2, b2 = ec.echo_rotary(plan, pos, q, k, stream=s)
    s.synchronize()
    assert (a == a2).all() and (b == b2).all()
    g, (a2, b2) = torch.cuda.CUDAGraph(), (torch.empty_like(q), torch.empty_like(k))
    with torch.cuda.graph(g):
        ec.echo_rotary(plan, pos, q, k, q_out=a2, k_out=b2)
    pos += 3
    g.replay()
    want, _ = ec.echo_rotary(plan, pos, q, k)
    assert (a2 == want).all() and not (a2 == a).all()
    n = ec.echo_launch_count()
    assert ec.echo_rotary(plan, pos[:0], q[:0], k[:0])[0].shape == (0, 256)
    assert ec.echo_launch_count() == n and ec.echo_get_device_error() == 0
