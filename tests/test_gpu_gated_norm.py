"""Norms around a gated residual against the oracle in fp64.

Tolerance, in units u = 2^-24 of fp32.  A sum over a row runs over at most 40 values of a
thread, 5 shuffles and 16 warps: off by 64 u of the sum of magnitudes, so a mean is off by 64 u
mean |v|, the mean of squares by (64 + 4) u of itself, the inverse root by half of that and 2
u (rsqrtf: 2 units of 2^-23): rel = 40 u together.  With m = mean |v| and r the inverse root, N(v) is off by
  rel |N| + 66 u r m (the mean's error, which the squares see again: twice, 132 u r m),
times |weight|, and each of weight, bias, gate, alpha, beta, 1 + scale and shift adds one rounding, u, of what it
makes: below 8 u of the sum S of the magnitudes of its terms.
h: 8 u S_h + beta gate off_after; n: the same of h's, through the norm (an error of e in h gives up to 3 r max e:
itself, the mean, the spread), and 8 u S_n.  Each is rounded once more: 2^-8 (bf16) or 2^-24 (fp32) of itself.
"""
import numpy as np
import pytest

pytestmark = pytest.mark.gpu

from oracle import norms as N                      # noqa: E402

F32 = np.float32
U = 2.0 ** -24


@pytest.fixture(scope="module")
def ec():
    import torch
    if not torch.cuda.is_available():
        pytest.skip("needs a GPU")
    from paper_2608_02474_gb300 import echocache
    return echocache


def rows(n, D, t, seed, wide=False):
    import torch
    x = np.random.default_rng(seed).standard_normal((n, D + (16 if wide else 0))).astype(F32)
    x[:, ::13] *= 6
    x += F32(0.7)
    x = torch.from_numpy(x).cuda().to(torch.bfloat16 if t == "bf16" else torch.float32)
    return x[:, :D]


def host(t):
    return None if t is None else t.float().cpu().numpy().astype(np.float64)


def norm_off(v, kind, weight, eps=1e-6):
    """(N without affine, its error)."""
    if kind == "none":
        return v, np.zeros_like(v)
    c = v - v.mean(axis=1, keepdims=True) if kind == "layer" else v
    r = 1 / np.sqrt((c * c).mean(axis=1, keepdims=True) + eps)
    m = np.abs(v).mean(axis=1, keepdims=True) if kind == "layer" else 0.0
    return c * r, (40 * U * np.abs(c) * r + 132 * U * r * m) * (1 if weight is None else np.abs(weight))


def check(got, x, y, gate, scale, shift, live, before="layer", weight=None, bias=None, after="none", after_weight=None,
          after_bias=None, alpha=1.0, beta=1.0, eps=1e-6):
    h, n = N.gated(x, y, gate, scale, shift, before, weight, bias, after, after_weight, after_bias, alpha, beta, eps)
    one = lambda a, b: 1.0 if a is None else np.abs(a) + b     # noqa: E731
    off_h, size_h = 0.0, np.abs(alpha * x)
    if y is not None:
        base, off = norm_off(y, after, after_weight, eps)
        ny = np.abs(base) * one(after_weight, 0) + (0 if after_bias is None else np.abs(after_bias))
        size_h = size_h + abs(beta) * one(gate, 0) * ny
        off_h = abs(beta) * one(gate, 0) * off
    off_h = off_h + 8 * U * size_h
    base, off = norm_off(h, before, weight, eps)
    c = h - h.mean(axis=1, keepdims=True) if before == "layer" else h
    r = 1.0 if before == "none" else 1 / np.sqrt((c * c).mean(axis=1, keepdims=True) + eps)
    through = off_h if before == "none" else 3 * r * off_h.max(axis=1, keepdims=True) * np.maximum(1, np.abs(base))
    nb = np.abs(base) * one(weight, 0) + (0 if bias is None else np.abs(bias))
    off_n = (off + through * one(weight, 0)) * one(scale, 1) + 8 * U * (nb * one(scale, 1) + (0 if shift is None else np.abs(shift)))
    for g, w, e in ((got[0], h, off_h), (got[1], n, off_n)):
        if g is None:
            continue
        half = 2.0 ** -8 if g.element_size() == 2 else U
        bad = np.abs(host(g) - w)[live] - (e + half * np.abs(w))[live]
        assert bad.max(initial=-1) <= 0, float(bad.max())


WIDTHS = [8, 64, 128, 256, 264, 512, 520, 1024, 1032, 2048, 2056, 4096, 4104, 5120, 5128, 8192, 8200, 12288, 12296, 16384]


@pytest.mark.parametrize("D", WIDTHS)
@pytest.mark.parametrize("after,before", [("none", "layer"), ("rms", "rms"), ("layer", "none")])
def test_widths(ec, D, after, before):
    import torch
    n, mods = 37, 5
    xt, yt, mt = [("bf16", "f32", "f32"), ("f32", "bf16", "bf16"), ("bf16", "bf16", "f32")][D // 8 % 3]
    x, y = rows(n, D, xt, D), rows(n, D, yt, D + 1, wide=True)
    table = rows(mods, 3 * D, mt, 5)
    gate, scale, shift = (table[:, i * D:(i + 1) * D] for i in range(3))
    m = np.random.default_rng(D).integers(0, mods, n)
    g = np.random.default_rng(3)
    w, b, aw = (torch.from_numpy(g.standard_normal(D).astype(F32)).cuda() for _ in range(3))
    plan = ec.GatedNorm(D, before, *((w, b) if before != "none" else (None, None)), after=after,
                        after_weight=aw if after != "none" else None, alpha=0.75, beta=-1.25)
    got = ec.echo_gated_norm(plan, x, y, gate, scale, shift, mod_rows=torch.from_numpy(m.astype(np.int32)).cuda(),
                             n=torch.empty(n, D, dtype=torch.float32 if D % 16 else torch.bfloat16, device="cuda"))
    check(got, host(x), host(y), host(gate)[m], host(scale)[m], host(shift)[m], slice(None), before,
          *((host(w), host(b)) if before != "none" else (None, None)), after, host(aw) if after != "none" else None,
          None, 0.75, -1.25)
    assert ec.echo_get_device_error() == 0


@pytest.mark.parametrize("n", [1, 2, 7, 8, 9, 1000, 20011])
@pytest.mark.parametrize("D", [64, 1024])
def test_numbers_of_rows(ec, n, D):
    """Rows by themselves and more than all blocks take at once; modulation by r // rows_per_mod."""
    x, y = rows(n, D, "bf16", n), rows(n, D, "bf16", n + 1)
    per = 3
    gate = rows((n + per - 1) // per, D, "f32", 2)
    m = np.arange(n) // per
    plan = ec.GatedNorm(D)
    got = ec.echo_gated_norm(plan, x, y, gate, rows_per_mod=per)
    check(got, host(x), host(y), host(gate)[m], None, None, slice(None))
    again = ec.echo_gated_norm(plan, x, y, gate, rows_per_mod=per)
    assert all((a == b).all() for a, b in zip(got, again))
    # a row's numbers are the same whatever the other rows
    one = ec.echo_gated_norm(plan, x[n // 2:n // 2 + 1], y[n // 2:n // 2 + 1], gate[n // 2 // per:], rows_per_mod=1)
    assert all((a[n // 2] == b[0]).all() for a, b in zip(got, one))


@pytest.mark.parametrize("D", [1032, 2048, 5120, 5128, 8192])
@pytest.mark.parametrize("after,before", [("none", "layer"), ("none", "none"), ("layer", "rms"), ("rms", "layer")])
@pytest.mark.parametrize("xt,yt", [("bf16", "bf16"), ("f32", "bf16"), ("f32", "f32")])
def test_many_rows(ec, D, after, before, xt, yt):
    """Rows that are copied ahead: sequences of modulations that change within and between
    batches, rows of none among them, in place, and the last rows of a block."""
    import torch
    n, mods = 4001, 9
    x, y = rows(n, D, xt, D), rows(n, D, yt, D + 1, wide=True)
    table = rows(mods, 3 * D, "f32", 5) / 4
    gate, scale, shift = (table[:, i * D:(i + 1) * D] for i in range(3))
    g = np.random.default_rng(D)
    m = np.sort(g.integers(0, mods, n))
    m[1000:1100] = g.integers(0, mods, 100)
    m[[5, 2000, 2001, 4000]] = [-1, mods, 2 ** 30, -2 ** 31]
    live = (m >= 0) & (m < mods)
    w, b = (torch.from_numpy(g.standard_normal(D).astype(F32)).cuda() for _ in range(2))
    plan = ec.GatedNorm(D, before, *((w, b) if before != "none" else (None, None)), after=after,
                        after_weight=b if after != "none" else None, alpha=1.5, beta=0.5)
    k = torch.full((n, D), 7.0, dtype=torch.bfloat16, device="cuda")
    xx = x.clone()
    mod = torch.from_numpy(m.astype(np.int32)).cuda()
    ec.echo_gated_norm(plan, xx, y, gate, scale, shift, mod_rows=mod, h=xx, n=k)
    again = ec.echo_gated_norm(plan, x, y, gate, scale, shift, mod_rows=mod)
    ok = torch.from_numpy(live)
    assert (xx[ok] == again[0][ok]).all() and (k[ok] == again[1][ok]).all()
    assert (xx[~ok] == x[~ok]).all() and (k[~ok] == 7.0).all()
    some = np.unique(np.concatenate([np.arange(30), np.arange(1000, 1100), np.arange(3950, n), g.integers(0, n, 60)]))
    at = torch.from_numpy(some).cuda()
    pick = lambda a: host(a)[np.where(live, m, 0)[some]]      # noqa: E731
    check((xx[at], k[at]), host(x[at]), host(y[at]), pick(gate), pick(scale), pick(shift), live[some], before,
          *((host(w), host(b)) if before != "none" else (None, None)), after, host(b) if after != "none" else None, None,
          1.5, 0.5)
    # without a branch, n or h alone, rows by number
    h, k = ec.echo_gated_norm(plan, x, scale=scale, shift=shift, rows_per_mod=500)
    mm = (some // 500)
    check((h[at], k[at]), host(x[at]), None, None, host(scale)[mm], host(shift)[mm], slice(None), before,
          *((host(w), host(b)) if before != "none" else (None, None)), "none", None, None, 1.5, 0.5)
    assert (ec.echo_gated_norm(plan, x, scale=scale, shift=shift, rows_per_mod=500, want_h=False)[1] == k).all()
    assert (ec.echo_gated_norm(plan, x, want_n=False)[0] == h).all()
    assert ec.echo_get_device_error() == 0


def test_parts(ec):
    """Without a branch, without gate, scale, shift; h or n alone; a norm alone is the layer norm."""
    import torch
    n, D = 20, 520
    x, y = rows(n, D, "f32", 1), rows(n, D, "f32", 2)
    plan = ec.GatedNorm(D, alpha=2.0)
    h, m = ec.echo_gated_norm(plan, x)
    check((h, m), host(x), None, None, None, None, slice(None), alpha=2.0)
    assert (h == 2 * x).all()
    a, none = ec.echo_gated_norm(plan, x, y, want_n=False)
    assert none is None
    check((a, None), host(x), host(y), None, None, None, slice(None), alpha=2.0)
    none, b = ec.echo_gated_norm(plan, x, y, want_h=False)
    assert none is None and (b == ec.echo_gated_norm(plan, x, y)[1]).all()
    for gate, scale, shift in ((None, y[:1], None), (None, None, y[:1]), (y[:1], None, None)):
        got = ec.echo_gated_norm(ec.GatedNorm(D, "rms"), x, y, gate, scale, shift, rows_per_mod=n)
        pick = lambda t: None if t is None else np.repeat(host(t), n, axis=0)    # noqa: E731
        check(got, host(x), host(y), pick(gate), pick(scale), pick(shift), slice(None), "rms")
    plain = ec.GatedNorm(D, "none")
    h, m = ec.echo_gated_norm(plain, x, n=torch.empty_like(x))
    assert (h == x).all() and (m == x).all()


def test_over_the_inputs(ec):
    """h in x's place, n in y's, and the other way round."""
    import torch
    n, D = 50, 2048
    x, y, gate = rows(n, D, "bf16", 1), rows(n, D, "bf16", 2), rows(n, D, "bf16", 3)
    plan = ec.GatedNorm(D, "rms", after="layer")
    h, m = ec.echo_gated_norm(plan, x, y, gate, rows_per_mod=1)
    for over_h, over_n in ((0, 1), (1, 0)):
        t = [x.clone(), y.clone()]
        ec.echo_gated_norm(plan, *t, gate, rows_per_mod=1, h=t[over_h], n=t[over_n])
        assert (t[over_h] == h).all() and (t[over_n] == m).all()
    assert torch.isfinite(m).all()


def test_rows_of_no_modulation(ec):
    """Rows whose number is no row of the table are left as they were."""
    import torch
    n, D = 30, 264
    x, y, gate = rows(n, D, "f32", 1), rows(n, D, "f32", 2), rows(4, D, "f32", 3)
    m = np.random.default_rng(4).integers(0, 4, n)
    m[[3, 29]], m[11], m[12] = -1, 4, 2 ** 31 - 1
    live = (m >= 0) & (m < 4)
    h, k = (torch.full((n, D), 5.0, device="cuda") for _ in range(2))
    ec.echo_gated_norm(ec.GatedNorm(D), x, y, gate, mod_rows=torch.from_numpy(m.astype(np.int32)).cuda(), h=h, n=k)
    check((h, k), host(x), host(y), host(gate)[np.where(live, m, 0)], None, None, live)
    assert (h[~torch.from_numpy(live)] == 5.0).all() and (k[~torch.from_numpy(live)] == 5.0).all()
    # r // rows_per_mod past the table
    h.fill_(5.0)
    ec.echo_gated_norm(ec.GatedNorm(D), x, y, gate, rows_per_mod=5, h=h)
    assert (h[20:] == 5.0).all() and not (h[:20] == 5.0).all(dim=1).any()


def test_not_finite(ec):
    """NaN and infinity stay in their rows."""
    n, D = 12, 1024
    x, y = rows(n, D, "bf16", 1), rows(n, D, "bf16", 2)
    x[3, 7], y[5, 1000] = float("nan"), float("inf")
    h, m = ec.echo_gated_norm(ec.GatedNorm(D), x, y)
    import torch
    ok = torch.isfinite(m).all(dim=1).tolist()
    assert ok == [i not in (3, 5) for i in range(n)]


def test_captured_and_streams(ec):
    import torch
    n, D = 64, 5120
    x, y, gate = rows(n, D, "f32", 1), rows(n, D, "bf16", 2), rows(n, D, "f32", 3)
    plan, mod = ec.GatedNorm(D), torch.arange(n, dtype=torch.int32, device="cuda")
    want = ec.echo_gated_norm(plan, x, y, gate, gate, gate, mod_rows=mod)
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    got = ec.echo_gated_norm(plan, x, y, gate, gate, gate, mod_rows=mod, stream=s)
    s.synchronize()
    assert all((a == b).all() for a, b in zip(got, want))
    h, m, g = torch.empty_like(x), torch.empty_like(want[1]), torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        ec.echo_gated_norm(plan, x, y, gate, gate, gate, mod_rows=mod, h=h, n=m)
    x *= 2
    g.replay()
    want = ec.echo_gated_norm(plan, x, y, gate, gate, gate, mod_rows=mod)
    assert (h == want[0]).all() and (m == want[1]).all()
    c = ec.echo_launch_count()
    assert ec.echo_gated_norm(plan, x[:0], y[:0])[0].shape == (0, D)
    assert ec.echo_launch_count() == c and ec.echo_get_device_error() == 0
