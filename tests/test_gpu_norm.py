"""Group norm with an activation against its definition in 64 bits.

Bounds, with u = 2^-24: a sum of n terms in fp32 in threads' runs and a tree is within C u of its
terms' sizes (C = 64 covers runs of that many).  x - mean carries u of |x|, so xhat and rstd are off by
at most T (1 + |xhat|) and T of themselves, T = C u (1 + max|x| rstd); an activation passes on at most
1.13 of an error of z and adds 4e-7 (1 + |z|) of its own, its slope 1.2 of it and the same.  Where relu
is closer to its corner than z's error, its slope counts as unknown."""
import numpy as np
import pytest
import torch

import layer_refs as ref
import paper_2507_16991_amd as mp

pytestmark = pytest.mark.gpu
DEV = torch.device("cuda:0")
U = 2.0 ** -24
C = 64
EPS = 1e-5
ROUND = {torch.float32: 2.0 ** -23, torch.bfloat16: 2.0 ** -8}


def lengths(n, s, kind, seed):
    r = np.random.default_rng(seed)
    if kind == "even":
        return np.array([n * i // s for i in range(s + 1)])
    cut = np.sort(r.integers(0, n + 1, s - 1))
    if kind == "skewed":  # one segment takes most
        cut = np.sort(r.integers(0, max(1, n // 8), s - 1))
        cut[s // 2:] += n - max(1, n // 8)
    return np.concatenate([[0], cut, [n]])


def spread(ptr, per_segment):
    """[S, ...] values to the segments' rows."""
    return np.repeat(per_segment, np.diff(ptr), axis=0)


def check(n, s, f, g, dtype, act="silu", kind="ragged", affine=True, offset=2.0, pad=0, ptr64=False,
          out_dtype=None, seed=1):
    gen = torch.Generator().manual_seed(seed)
    x = torch.randn(n, f + pad, generator=gen)
    x = (x * (0.5 + torch.rand(f + pad, generator=gen)) + offset * torch.randn(f + pad, generator=gen))
    x = x.to(dtype).to(DEV)[:, :f]
    dout = torch.randn(n, f, generator=gen).to(dtype).to(DEV)
    weight = (1 + 0.2 * torch.randn(f, generator=gen)).to(DEV) if affine else None
    bias = (0.3 * torch.randn(f, generator=gen)).to(DEV) if affine else None
    p = lengths(n, s, kind, seed)
    ptr = torch.from_numpy(p.astype(np.int64 if ptr64 else np.int32)).to(DEV)
    w64 = ref.f64(weight) if affine else np.ones(f)
    r = ref.group_norm(p, ref.f64(x), g, w64, ref.f64(bias) if affine else np.zeros(f), EPS, act)

    out, mean, rstd = mp.group_norm(ptr, x, g, weight=weight, bias=bias, eps=EPS, act=act,
                                    out_dtype=out_dtype)
    cg = f // g
    big = np.zeros((s, g))
    for i in range(s):
        if p[i] < p[i + 1]:
            big[i] = np.abs(ref.f64(x)[p[i]:p[i + 1]]).reshape(-1, g, cg).max((0, 2))
    T = C * U * (1 + big * r["rstd"])
    assert np.all(np.abs(ref.f64(mean) - r["mean"]) <= C * U * big)
    assert np.all(np.abs(ref.f64(rstd) - r["rstd"]) <= T * r["rstd"])
    Tx = np.repeat(spread(p, T), cg, axis=1)
    zerr = np.abs(w64) * Tx * (1 + np.abs(r["xhat"])) + 4 * U * np.abs(r["z"])
    own = 4e-7 * (1 + np.abs(r["z"]))
    rounding = ROUND[out.dtype]
    assert np.all(np.abs(ref.f64(out) - r["out"]) <= 1.13 * zerr + own + rounding * np.abs(r["out"]))

    dx, dw, db = mp.group_norm_backward(ptr, x, dout, g, mean, rstd, weight=weight, bias=bias, act=act)
    dx_r, dw_r, db_r = ref.group_norm_backward(p, r, ref.f64(dout), g, w64, act)
    d = np.abs(ref.f64(dout))
    slope_err = 1.2 * zerr + own + ((np.abs(r["z"]) <= zerr) if act == "relu" else 0)
    da_err = d * slope_err + 4 * U * d * 1.13
    da = d * 1.13
    xh = np.abs(r["xhat"])
    # sums over rows: the terms' errors and the summation's
    assert np.all(np.abs(ref.f64(db) - db_r) <= (da_err + C * U * da).sum(0))
    term = da_err * xh + da * Tx * (1 + xh)
    assert np.all(np.abs(ref.f64(dw) - dw_r) <= (term + C * U * da * xh).sum(0))
    bound = np.zeros((n, f))
    wa = np.abs(w64)
    for i in range(s):
        a, b = p[i], p[i + 1]
        if a == b:
            continue
        def over(v):
            return np.repeat(v[a:b].reshape(-1, g, cg).mean((0, 2)), cg)
        m1, e1 = over(wa * da), over(wa * (da_err + C * U * da))
        m2, e2 = over(wa * da * xh), over(wa * (term + C * U * da * xh))
        t = Tx[a:b]
        size = wa * da[a:b] + m1 + xh[a:b] * m2
        err = wa * da_err[a:b] + e1 + xh[a:b] * e2 + t * (1 + xh[a:b]) * m2
        bound[a:b] = np.repeat(r["rstd"][i], cg) * (err + (t + 8 * U) * size)
    rounding = ROUND[dx.dtype]
    assert np.all(np.abs(ref.f64(dx) - dx_r) <= bound + rounding * np.abs(dx_r))


DTYPES = [torch.float32, torch.bfloat16]


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("n,s,f,g", [(1, 1, 1, 1), (1, 1, 8, 8), (3, 2, 5, 5), (7, 3, 3, 1),
                                     (50, 9, 12, 3), (200, 30, 13, 1), (333, 20, 64, 8),
                                     (500, 37, 100, 4), (400, 3, 128, 32), (1000, 1, 100, 10),
                                     (900, 300, 129, 3), (64, 5, 520, 8), (2708, 1, 64, 8)])
def test_sizes(n, s, f, g, dtype):
    check(n, s, f, g, dtype)


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("act", ["none", "relu", "silu", "gelu"])
@pytest.mark.parametrize("affine", [True, False])
def test_activations(act, affine, dtype):
    check(700, 11, 48, 6, dtype, act=act, affine=affine)


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("n,s,f,g,kind", [(20000, 40, 32, 4, "skewed"), (20011, 3, 100, 4, "even"),
                                          (30001, 3000, 16, 16, "skewed"), (9000, 7, 129, 3, "ragged"),
                                          (12000, 100, 6, 2, "skewed"), (5000, 2, 300, 300, "even")])
def test_long_segments(n, s, f, g, kind, dtype):
    check(n, s, f, g, dtype, act="gelu", kind=kind)


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("n,s,f,g", [(9, 3, 4096, 8), (7, 2, 2051, 7), (40, 3, 3000, 3000),
                                     (200, 2, 8192, 64), (5, 2, 16384, 64), (4, 3, 16390, 2),
                                     (6, 2, 20000, 1), (3, 1, 65536, 4), (2, 2, 65535, 65535)])
def test_wide_rows(n, s, f, g, dtype):
    check(n, s, f, g, dtype)


@pytest.mark.parametrize("dtype", DTYPES)
def test_strides_and_index_types(dtype):
    check(600, 20, 60, 4, dtype, pad=7, ptr64=True)
    check(6000, 2, 60, 4, dtype, pad=4, ptr64=True, kind="skewed")
    check(300, 5, 64, 8, dtype, out_dtype=torch.float32)


def test_mean_large_against_the_spread():
    """Rows near 1000 with a spread of 1: the variance keeps its digits on both paths."""
    for n, s in ((400, 10), (30000, 2)):
        check(n, s, 32, 4, torch.float32, offset=1000.0)


def test_constant_rows_and_outliers():
    for n in (100, 20000):
        x = torch.full((n, 16), 3.25, device=DEV)
        ptr = torch.tensor([0, n], dtype=torch.int32, device=DEV)
        out, mean, rstd = mp.group_norm(ptr, x, 4)
        assert bool((out == 0).all()) and bool((mean == 3.25).all())
        assert torch.allclose(rstd, torch.full_like(rstd, EPS ** -0.5), rtol=1e-6, atol=0)
        x = torch.randn(n, 16, device=DEV)
        x[0] = 1e6  # a first row that is no sample of the others
        _, mean, rstd = mp.group_norm(ptr, x, 4)
        v = x.double().view(n, 4, 4)
        m = v.mean((0, 2))
        want = 1 / ((v - m[:, None]).square().mean((0, 2)) + EPS).sqrt()
        assert torch.allclose(rstd[0].double(), want, rtol=1e-5, atol=0)


def test_empty_segments():
    for n, p in ((0, [0, 0, 0]), (5, [0, 0, 5, 5]), (20000, [0, 0, 0, 20000, 20000])):
        x = torch.randn(n, 8, device=DEV)
        ptr = torch.tensor(p, dtype=torch.int32, device=DEV)
        out, mean, rstd = mp.group_norm(ptr, x, 2)
        empty = (ptr[1:] == ptr[:-1])
        assert bool((mean[empty] == 0).all()) and bool((rstd[empty] == 0).all())
        assert bool((rstd[~empty] > 0).all()) and out.shape == x.shape
        dx, dw, db = mp.group_norm_backward(ptr, x, x, 2, mean, rstd)
        assert torch.allclose(db, x.sum(0), atol=1e-2)
        if n == 0:
            assert bool((dw == 0).all()) and bool((db == 0).all())
    x = torch.empty(0, 20000, device=DEV)  # (groups too wide for the short path)
    ptr = torch.zeros(4, dtype=torch.int32, device=DEV)
    _, mean, rstd = mp.group_norm(ptr, x, 1)
    assert bool((mean == 0).all()) and bool((rstd == 0).all())


def test_parts_of_the_gradient():
    x = torch.randn(3000, 24, device=DEV)
    d = torch.randn(3000, 24, device=DEV)
    ptr = torch.tensor([0, 100, 3000], dtype=torch.int32, device=DEV)
    _, mean, rstd = mp.group_norm(ptr, x, 3, act="silu")
    dx, dw, db = mp.group_norm_backward(ptr, x, d, 3, mean, rstd, act="silu")
    a = mp.group_norm_backward(ptr, x, d, 3, mean, rstd, act="silu", want_dw=False)
    b = mp.group_norm_backward(ptr, x, d, 3, mean, rstd, act="silu", want_dx=False)
    assert a[1] is None and a[2] is None and b[0] is None
    assert torch.equal(a[0], dx) and torch.equal(b[1], dw) and torch.equal(b[2], db)


@pytest.mark.parametrize("act", ["none", "silu", "gelu"])
def test_gradient_against_differences(act):
    """The kernel's gradient against central differences of the definition in 64 bits."""
    r = np.random.default_rng(3)
    p = np.array([0, 4, 4, 9])
    x, d = r.standard_normal((9, 6)), r.standard_normal((9, 6))
    w, b = 1 + 0.2 * r.standard_normal(6), 0.1 * r.standard_normal(6)
    x, d, w, b = (v.astype(np.float32) for v in (x, d, w, b))

    def f(x, w, b):
        return (ref.group_norm(p, x, 2, w, b, EPS, act)["out"] * d).sum()

    def diff(i, v):
        h, out = 1e-5, np.zeros(v.shape)
        for j in np.ndindex(v.shape):
            args = [a.astype(np.float64) for a in (x, w, b)]
            args[i][j] += h
            hi = f(*args)
            args[i][j] -= 2 * h
            out[j] = (hi - f(*args)) / (2 * h)
        return out

    t = [torch.from_numpy(v).to(DEV) for v in (x, d, w, b)]
    ptr = torch.from_numpy(p).to(DEV)
    _, mean, rstd = mp.group_norm(ptr, t[0], 2, weight=t[2], bias=t[3], act=act)
    got = mp.group_norm_backward(ptr, t[0], t[1], 2, mean, rstd, weight=t[2], bias=t[3], act=act)
    for i, (g, v) in enumerate(zip(got, (x, w, b))):
        assert np.abs(ref.f64(g) - diff(i, v)).max() < 2e-5


def test_same_inputs_same_bits_and_side_stream():
    x = torch.randn(30000, 40, device=DEV)
    ptr = torch.tensor([0, 50, 60, 25000, 30000], dtype=torch.int32, device=DEV)
    torch.cuda.synchronize()
    s = torch.cuda.Stream()
    a = mp.group_norm(ptr, x, 4, act="gelu")
    b = mp.group_norm(ptr, x, 4, act="gelu", stream=s)
    torch.cuda.synchronize()
    for u, v in zip(a, b):
        assert torch.equal(u, v)
    ga = mp.group_norm_backward(ptr, x, x, 4, a[1], a[2], act="gelu")
    gb = mp.group_norm_backward(ptr, x, x, 4, a[1], a[2], act="gelu", stream=s)
    torch.cuda.synchronize()
    for u, v in zip(ga, gb):
        assert torch.equal(u, v)


def test_refusals():
    x = torch.randn(4, 8, device=DEV)
    ptr = torch.tensor([0, 4], dtype=torch.int32, device=DEV)
    for groups in (0, 3, 9):
        with pytest.raises(mp.MPError):
            mp.group_norm(ptr, x, groups)
    with pytest.raises(mp.MPError):
        mp.group_norm(ptr, x, 2, eps=-1.0)
    with pytest.raises(mp.MPError):
        mp.group_norm(ptr[:1], x, 2)
    with pytest.raises(ValueError):
        mp.group_norm(ptr, x, 2, act="tanh")
    with pytest.raises(ValueError):
        mp.group_norm(ptr, x, 2, weight=torch.ones(7, device=DEV))
    with pytest.raises(ValueError):
        mp.group_norm(ptr.float(), x, 2)
    with pytest.raises(ValueError):
        mp.group_norm(ptr, x.t(), 2)
    _, mean, rstd = mp.group_norm(ptr, x, 2)
    with pytest.raises(ValueError):
        mp.group_norm_backward(ptr, x, x.bfloat16(), 2, mean, rstd)
    with pytest.raises(ValueError):
        mp.group_norm_backward(ptr, x, x, 2, mean, rstd[:, :1])
    with pytest.raises(mp.MPError):
        mp.group_norm_backward(ptr, x, x, 2, mean, rstd, want_dx=False, want_dw=False)
