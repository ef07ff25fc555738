"""Root-mean-square norm, its 8-bit result and its gradients against their definitions in 64 bits."""
import numpy as np
import pytest
import torch

import paper_2507_16991_amd as mp
import row_refs as ref
from layer_refs import f64

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
F32, BF16 = torch.float32, torch.bfloat16
EPS = 1e-5

# A thread adds at most 64 squares, a wavefront's 6 and a workgroup's 16 sums follow: the relative error of
# the sum of squares is 87 half steps (with the square's), of the mean and with eps 89, of its root 45, of
# rstd 47; out takes two products more.
RSTD = 47 * ref.U
OUT = 49 * ref.U

SHAPES = [(1, 1), (3, 2), (5, 3), (4, 5), (7, 8), (9, 31), (130, 64), (33, 100), (2, 127), (65, 256), (3, 511),
          (5, 513), (9, 1000), (3, 1026), (2, 2047), (3, 2050), (2, 4096), (3, 8191), (2, 16384), (2, 20003),
          (1, 32769), (2, 65536)]


def randn(seed, *shape, dtype=F32):
    return torch.randn(*shape, generator=torch.Generator().manual_seed(seed)).to(dtype).to(DEV)


def check_out(total, weight, out, rstd, eps=EPS):
    want, r, _ = ref.rms_norm(f64(total), 1.0 if weight is None else f64(weight), eps)
    assert (np.abs(f64(rstd) - r) <= r * RSTD).all()
    tol = np.abs(want) * (OUT + (ref.half_step(BF16) * 1.01 if out.dtype == BF16 else 0))
    assert (np.abs(f64(out) - want) <= tol).all()


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("n,f", SHAPES)
def test_norm(n, f, dtype):
    x, res, w = randn(1, n, f, dtype=dtype), randn(2, n, f, dtype=dtype), randn(3, f)
    out, total, rstd = mp.rms_norm(x, w, eps=EPS)
    assert total is x
    check_out(x, w, out, rstd)
    out, total, rstd = mp.rms_norm(x, w, residual=res, eps=EPS)
    assert torch.equal(total, x + res)  # (one rounding, as torch's)
    check_out(total, w, out, rstd)


@pytest.mark.parametrize("dtype,out", [(F32, BF16), (BF16, F32)])
def test_other_output_type_and_no_weight(dtype, out):
    x = randn(4, 37, 300, dtype=dtype)
    y, _, rstd = mp.rms_norm(x, eps=EPS, out_dtype=out)
    assert y.dtype == out
    check_out(x, None, y, rstd)


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("n,f", SHAPES)
def test_gradients(n, f, dtype):
    x, d, dt, w = (randn(5, n, f, dtype=dtype), randn(6, n, f, dtype=dtype), randn(7, n, f, dtype=dtype),
                   randn(8, f))
    _, _, rstd = mp.rms_norm(x, w, eps=EPS)
    for dtotal in (None, dt):
        dx, dw = mp.rms_norm_backward(x, d, rstd, w, dtotal=dtotal)
        want, size, wdw, sdw = ref.rms_norm_backward(f64(x), f64(d), f64(w), EPS,
                                                     None if dtotal is None else f64(dtotal))
        # rstd enters three times (its own, xhat, the mean's xhat); the mean is a sum as above (88), and
        # eight roundings more
        tol = size * (3 * 47 + 88 + 8) * ref.U
        tol = tol + (np.abs(want) + tol) * (ref.half_step(BF16) if dtype == BF16 else 0)
        assert (np.abs(f64(dx) - want) <= tol).all()
        # n additions, the product and xhat
        assert (np.abs(f64(dw) - wdw) <= sdw * (n + 50) * ref.U).all()


def test_gradients_of_many_rows():
    x, d, w = randn(1, 70001, 36), randn(2, 70001, 36), randn(3, 36)
    _, _, rstd = mp.rms_norm(x, w)
    dx, dw = mp.rms_norm_backward(x, d, rstd, w)
    want, size, wdw, sdw = ref.rms_norm_backward(f64(x), f64(d), f64(w), EPS)
    assert (np.abs(f64(dx) - want) <= size * 237 * ref.U).all()
    # 5 rows a team, 16 teams of a workgroup, 32 of 1,024 workgroups a thread, 32 threads
    assert (np.abs(f64(dw) - wdw) <= sdw * (5 + 16 + 32 + 32 + 50) * ref.U).all()
    only = mp.rms_norm_backward(x, d, rstd, w, want_dw=False)
    assert only[1] is None and torch.equal(only[0], dx)
    only = mp.rms_norm_backward(x, d, rstd, w, want_dx=False)
    assert only[0] is None and torch.equal(only[1], dw)


def test_wide_rows_of_many():
    x, d, w = randn(1, 2050, 20000, dtype=BF16), randn(2, 2050, 20000, dtype=BF16), randn(3, 20000)
    _, _, rstd = mp.rms_norm(x, w)
    dx, dw = mp.rms_norm_backward(x, d, rstd, w, dx_dtype=F32)
    want, size, wdw, sdw = ref.rms_norm_backward(f64(x), f64(d), f64(w), EPS)
    assert (np.abs(f64(dx) - want) <= size * 237 * ref.U).all()
    assert (np.abs(f64(dw) - wdw) <= sdw * (2050 + 50) * ref.U).all()


def test_gradient_by_differences():
    """The derivative of sum(dout * out) along a direction, in 64 bits, by central differences."""
    x, d, w, v = randn(1, 6, 90), randn(2, 6, 90), randn(3, 90), randn(4, 6, 90)
    _, _, rstd = mp.rms_norm(x, w)
    dx, _ = mp.rms_norm_backward(x, d, rstd, w)
    h = 1e-5
    up, down = (ref.rms_norm(f64(x) + s * h * f64(v), f64(w), EPS)[0] for s in (1, -1))
    slope = ((up - down) * f64(d)).sum() / (2 * h)
    size = ref.rms_norm_backward(f64(x), f64(d), f64(w), EPS)[1]
    # the kernel's rounding, and the differences' h^2 (third derivatives of order one) and 2^-52 / h
    assert abs(float((dx.double() * v.double()).sum()) - slope) <= float((size * np.abs(f64(v))).sum()) * (
        237 * ref.U + 1e-9)


def quantized(x, w, res=None, total=None):
    n, f = x.shape
    kb = -(-f // 32)
    codes = torch.full((n, 32 * kb), 99, dtype=torch.uint8, device=DEV)
    scales = torch.full((n, kb), 99, dtype=torch.uint8, device=DEV)
    values = torch.empty(n, f, dtype=x.dtype, device=DEV)
    rstd = torch.empty(n, device=DEV)
    dt = mp.MP_F32 if x.dtype == F32 else mp.MP_BF16
    mp.mp_rms_norm_mx8(x, dt, n, f, f, res, f, w, EPS, total, codes, scales, values, rstd)
    return codes, scales, values, rstd


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("n,f", SHAPES)
def test_eight_bits(n, f, dtype):
    x, res, w = randn(1, n, f, dtype=dtype), randn(2, n, f, dtype=dtype), randn(3, f)
    w *= torch.exp2(4 * randn(4, f))
    total = torch.empty_like(x)
    codes, scales, values, rstd = quantized(x, w, res, total)
    assert torch.equal(total, x + res)
    _, r, _ = ref.rms_norm(f64(total), 1.0, EPS)
    assert (np.abs(f64(rstd) - r) <= r * RSTD).all()
    # from rstd on two products rounded to fp32: the same in numpy
    v = (total.float().cpu().numpy() * rstd.cpu().numpy()[:, None]).astype(np.float32)
    v = (v * w.cpu().numpy()).astype(np.float32).astype(np.float64)
    code, s = ref.mx8_quantize(v)
    assert np.array_equal(scales.cpu().numpy().astype(np.int64), s)
    assert np.array_equal(codes.cpu().numpy().reshape(code.shape).astype(np.int64), code)
    assert np.array_equal(f64(values), ref.mx8_values(code, s)[:, :f])
    assert torch.equal(mp.mx8_dequantize(codes, scales, f, dtype=dtype), values)
    c2, s2, v2, t2 = mp.rms_norm_mx8(x, w, residual=res, eps=EPS, want_values=True)
    assert torch.equal(c2, codes) and torch.equal(s2, scales) and torch.equal(v2, values) and torch.equal(t2, total)


def test_every_code():
    codes = torch.arange(256, device=DEV).repeat(2).view(2, 256).to(torch.uint8)
    scales = torch.tensor([[127, 0, 1, 254, 255, 100, 7, 128]] * 2, dtype=torch.uint8, device=DEV)
    got = f64(mx := mp.mx8_dequantize(codes, scales, 256))
    want = ref.mx8_values(np.tile(np.arange(256), (2, 1)).reshape(2, 8, 32), scales.cpu().numpy().astype(np.int64))
    with np.errstate(over="ignore"):
        want = want.astype(np.float32).astype(np.float64)
    assert np.array_equal(got, want, equal_nan=True), mx


def test_extreme_rows():
    """Squares that overflow, tiny ones, zeros, infinities and NaN, each in a row of its own."""
    f = 200
    x = randn(1, 8, f)
    x[1] *= 1e30
    x[2] = 0
    x[3] *= 1e-30
    x[4] *= 2e37
    x[5, 7] = float("inf")
    x[6, 3] = float("nan")
    out, _, rstd = mp.rms_norm(x, eps=EPS)
    good = [0, 1, 2, 3, 4, 7]
    want, r, _ = ref.rms_norm(f64(x)[good], 1.0, EPS)
    assert (np.abs(f64(rstd)[good] - r) <= r * RSTD + 2.0 ** -149).all()
    # (an rstd below the normal numbers, of rows around 2^127, is off by half a subnormal step)
    tol = np.abs(want) * OUT + np.abs(f64(x)[good]) * 2.0 ** -149
    assert (np.abs(f64(out)[good] - want) <= tol).all()
    o = f64(out)
    assert np.isnan(o[5, 7]) and (np.delete(o[5], 7) == 0).all() and np.isnan(o[6]).all()
    codes, scales, values, _ = mp.rms_norm_mx8(x, eps=EPS, want_values=True)
    bad = np.isnan(f64(values))
    assert bad[6].all() and bad[5, :32].all() and not bad[5, 32:].any() and not bad[good].any()
    assert (scales[2] == 0).all() and (codes[2] == 0).all()


def test_smallest_eps():
    x = randn(1, 4, 77) * 1e-20
    eps = float(torch.finfo(F32).tiny)
    out, _, rstd = mp.rms_norm(x, eps=eps)
    # every square is off by half of 2^-149 at most, the mean thus by 2^-150, and eps is 2^-126
    want, r, _ = ref.rms_norm(f64(x), 1.0, eps)
    assert (np.abs(f64(rstd) - r) <= r * (RSTD + 2.0 ** -24)).all()
    assert (np.abs(f64(out) - want) <= np.abs(want) * (OUT + 2.0 ** -24)).all()


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("f", [5, 100, 257, 2051, 9000])
def test_in_place_total_and_strided_rows(f, dtype):
    x, res, w = randn(1, 41, f, dtype=dtype), randn(2, 41, f, dtype=dtype), randn(3, f)
    out, total, rstd = mp.rms_norm(x, w, residual=res)
    wide_x, wide_r = torch.zeros(41, f + 7, dtype=dtype, device=DEV), torch.zeros(41, f + 3, dtype=dtype, device=DEV)
    wide_x[:, 1:f + 1], wide_r[:, 2:f + 2] = x, res
    o2, t2, r2 = mp.rms_norm(wide_x[:, 1:f + 1], w, residual=wide_r[:, 2:f + 2])
    assert torch.equal(o2, out) and torch.equal(t2, total) and torch.equal(r2, rstd)
    d = randn(5, 41, f, dtype=dtype)
    wide_t = torch.zeros(41, f + 5, dtype=dtype, device=DEV)
    wide_t[:, 3:f + 3] = total
    for a, b in zip(mp.rms_norm_backward(wide_t[:, 3:f + 3], d, rstd, w), mp.rms_norm_backward(total, d, rstd, w)):
        assert torch.equal(a, b)
    q = mp.rms_norm_mx8(x, w, residual=res)
    xs, rs = x.clone(), res.clone()
    for over in (xs, rs):
        o2, t2, _ = mp.rms_norm(xs if over is xs else x, w, residual=rs if over is rs else res, total=over)
        assert t2 is over and torch.equal(over, total) and torch.equal(o2, out)
    rs.copy_(res)
    q2 = mp.rms_norm_mx8(x, w, residual=rs, total=rs)
    assert torch.equal(q2[0], q[0]) and torch.equal(q2[1], q[1]) and torch.equal(rs, total)


def test_no_rows():
    x = torch.empty(0, 40, device=DEV)
    out, total, rstd = mp.rms_norm(x)
    dx, dw = mp.rms_norm_backward(x, x, rstd)
    assert out.shape == dx.shape == (0, 40) and not dw.any()
    wide = torch.empty(0, 60000, device=DEV)
    assert not mp.rms_norm_backward(wide, wide, rstd)[1].any()
    assert mp.rms_norm_mx8(x)[0].shape == (0, 64)


def test_replayed_from_a_graph():
    x, res, d, w = randn(1, 3000, 96, dtype=BF16), randn(2, 3000, 96, dtype=BF16), randn(3, 3000, 96, dtype=BF16), randn(4, 96)

    def step():
        out, total, rstd = mp.rms_norm(x, w, residual=res)
        return out, total, *mp.rms_norm_backward(total, d, rstd, w, dtotal=d), *mp.rms_norm_mx8(x, w)[:2]

    step()
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        got = step()
    for seed in range(3):
        x.copy_(randn(10 + seed, 3000, 96, dtype=BF16))
        d.copy_(randn(20 + seed, 3000, 96, dtype=BF16))
        g.replay()
        torch.cuda.synchronize()
        for a, b in zip(got, step()):
            assert torch.equal(a, b)


def test_other_stream():
    x, res = randn(1, 500, 700), randn(2, 500, 700)
    want = mp.rms_norm(x, residual=res)
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    got = mp.rms_norm(x, residual=res, stream=s)
    torch.cuda.current_stream().wait_stream(s)
    for a, b in zip(got, want):
        assert torch.equal(a, b)


def test_tables_past_32_bits():
    n, f = 40001, 65536
    x = torch.zeros(n, f, dtype=BF16, device=DEV)
    assert x.numel() > 2 ** 31
    rows = torch.tensor([0, 32767, 32768, 32769, n - 1], device=DEV)
    x[rows] = randn(1, 5, f, dtype=BF16)
    out, _, rstd = mp.rms_norm(x)
    few = mp.rms_norm(x[rows])
    assert torch.equal(out[rows], few[0]) and torch.equal(rstd[rows], few[2])
    assert int((out != 0).any(1).sum()) == 5
    dx, dw = mp.rms_norm_backward(x, out, rstd)
    fdx, fdw = mp.rms_norm_backward(x[rows], few[0], few[2])
    assert torch.equal(dx[rows], fdx)
    # (all other rows add zeros: five additions in another order)
    assert (np.abs(f64(dw) - f64(fdw)) <= 2 * 5 * ref.U * np.abs(f64(x[rows]) * f64(few[2])[:, None]
                                                                * f64(few[0])).sum(0)).all()


def test_two_streams_at_once():
    a, b = randn(1, 20000, 300), randn(2, 9000, 1000, dtype=BF16)
    want = mp.rms_norm_backward(a, a, mp.rms_norm(a)[2]), mp.rms_norm_backward(b, b, mp.rms_norm(b)[2])
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    for _ in range(3):
        one = mp.rms_norm_backward(a, a, mp.rms_norm(a, stream=s)[2], stream=s)
        two = mp.rms_norm_backward(b, b, mp.rms_norm(b)[2])
        torch.cuda.synchronize()
        for x, y in zip((*one, *two), (*want[0], *want[1])):
            assert torch.equal(x, y)
