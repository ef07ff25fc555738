"""Microscaled 4-bit floating point: quantisation is exact against the definition; a product's terms
are exact in fp32, so its error is that of at most K additions, each within 2^-23 of the sizes added
so far, of which a step of the matrix cores makes few."""
import numpy as np
import pytest
import torch

import layer_refs as ref
import paper_2507_16991_amd as mp

pytestmark = pytest.mark.gpu
DEV = torch.device("cuda:0")
DTYPES = [torch.float32, torch.bfloat16]


def rows(n, k, dtype, seed, pad=0):
    g = torch.Generator().manual_seed(seed)
    x = torch.randn(n, k + pad, generator=g) * torch.exp2(3 * torch.randn(n, 1, generator=g))
    x[torch.rand(n, k + pad, generator=g) < 0.01] *= 50
    return x.to(dtype).to(DEV)[:, :k]


def check_quantize(x):
    codes, scales, values = mp.mx_quantize(x, want_values=True)
    code, s, value = ref.mx_quantize(ref.f64(x))
    assert np.array_equal(scales.cpu().numpy(), s)
    good = np.repeat(s != 255, 16, axis=-1)
    assert np.array_equal(codes.cpu().numpy()[good], ref.mx_pack(code)[good])
    assert values.dtype == x.dtype and np.array_equal(ref.f64(values), value, equal_nan=True)
    for dtype in DTYPES:
        back = mp.mx_dequantize(codes, scales, x.shape[1], dtype=dtype)
        assert back.dtype == dtype and np.array_equal(ref.f64(back), value, equal_nan=True)
    c, z = mp.mx_quantize(x)
    assert torch.equal(c, codes) and torch.equal(z, scales)


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("n,k", [(1, 1), (1, 31), (3, 32), (5, 33), (70, 64), (33, 100), (9, 1000),
                                 (2, 4100), (1, 65536), (1000, 8), (257, 130)])
def test_quantize(n, k, dtype):
    check_quantize(rows(n, k, dtype, n + k))


@pytest.mark.parametrize("dtype", DTYPES)
def test_quantize_strided_rows(dtype):
    check_quantize(rows(40, 77, dtype, 1, pad=5))


@pytest.mark.parametrize("dtype", DTYPES)
def test_quantize_ties_ranges_and_specials(dtype):
    """Halfway points of every step, saturation, signed zeros, the smallest and largest magnitudes, and
    blocks that hold an infinity or NaN."""
    steps = [0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5.0, 6.5, 7.0, 7.5, 0.0, 0.5, 1.0, 2.0, 3.0, 4.0, 6.0]
    line = torch.zeros(32)
    line[:17] = torch.tensor(steps)
    line[17:] = -line[2:17]
    line[31] = 4.0  # so that the block's scale is 1
    x = torch.stack([line * 2.0 ** e for e in range(-133, 124, 4)])
    specials = torch.zeros(8, 32)
    specials[0, 3] = float("inf")
    specials[1, 4] = float("-inf")
    specials[2, 31] = float("nan")
    specials[3, :] = -0.0
    specials[4, 0] = torch.finfo(dtype).max
    specials[5, 0] = torch.finfo(dtype).tiny
    specials[6, 0] = 1e-40
    specials[7, :5] = torch.tensor([1.0, -1.0, float("nan"), 2.0, 3.0])
    x = torch.cat([x, specials])
    check_quantize(torch.cat([x, x.flip(0)], 1).to(dtype).to(DEV))


def segments(n, t, kind, seed):
    r = np.random.default_rng(seed)
    if kind == "even":
        return np.array([n * i // t for i in range(t + 1)])
    if kind == "one":  # all rows in one segment
        at = int(r.integers(0, t))
        return np.array([0] * (at + 1) + [n] * (t - at))
    return np.concatenate([[0], np.sort(r.integers(0, n + 1, t - 1)), [n]])


def weights(t, fo, k, seed):
    """Random codes under scales of a few powers of two, in the format's layout."""
    r = np.random.default_rng(seed)
    kb = -(-k // 32)
    code = r.integers(0, 16, (t, fo, kb, 32))
    code.reshape(t, fo, -1)[:, :, k:] = 0
    s = r.integers(118, 130, (t, fo, kb))
    return code, s


def check_product(n, t, k, fo, x_dtype=torch.bfloat16, out_dtype=torch.float32, kind="ragged", pad=0,
                  seg64=False, seed=3):
    x = rows(n, k, x_dtype, seed, pad)
    p = segments(n, t, kind, seed)
    code, s = weights(t, fo, k, seed)
    seg = torch.from_numpy(p.astype(np.int64 if seg64 else np.int32)).to(DEV)
    codes = torch.from_numpy(ref.mx_pack(code)).to(DEV)
    scales = torch.from_numpy(s.astype(np.uint8)).to(DEV)
    out = mp.mx_segment_matmul(seg, x, codes, scales, out_dtype=out_dtype)
    w = ref.mx_values(code, s).reshape(t, fo, -1)[:, :, :k]
    v = ref.mx_quantize(ref.f64(x))[2]
    want, size = np.zeros((n, fo)), np.zeros((n, fo))
    for i in range(t):
        a, b = p[i], p[i + 1]
        want[a:b] = v[a:b] @ w[i].T
        size[a:b] = np.abs(v[a:b]) @ np.abs(w[i]).T
    rounding = 2.0 ** -8 if out_dtype == torch.bfloat16 else 0.0
    bound = (k / 32 + 16) * 2.0 ** -23 * size + rounding * np.abs(want)
    assert out.dtype == out_dtype and np.all(np.abs(ref.f64(out) - want) <= bound)
    return x, seg, codes, scales, out


@pytest.mark.parametrize("x_dtype", DTYPES)
@pytest.mark.parametrize("out_dtype", DTYPES)
@pytest.mark.parametrize("n,t,k,fo", [(1, 1, 1, 1), (1, 8, 64, 64), (1, 1, 4096, 33), (7, 3, 100, 17),
                                      (16, 8, 256, 100), (40, 2, 31, 40), (130, 1, 128, 128),
                                      (300, 5, 128, 128), (513, 4, 96, 200), (1000, 3, 544, 72),
                                      (2000, 64, 64, 128), (777, 2, 1000, 300)])
def test_product(n, t, k, fo, x_dtype, out_dtype):
    check_product(n, t, k, fo, x_dtype, out_dtype)


@pytest.mark.parametrize("n,t,k,fo,kind", [(5000, 3, 256, 4096, "even"), (17000, 5, 288, 1030, "ragged"),
                                           (9000, 2, 800, 2048, "one"), (70000, 1, 64, 256, "even"),
                                           (3, 4096, 64, 32, "ragged"), (20000, 300, 40, 24, "ragged"),
                                           (300, 3, 20000, 64, "ragged")])
def test_product_large(n, t, k, fo, kind):
    check_product(n, t, k, fo, out_dtype=torch.bfloat16, kind=kind)


def test_product_strides_and_index_types():
    check_product(333, 4, 100, 48, pad=9, seg64=True)
    check_product(333, 4, 100, 48, torch.float32, pad=3, seg64=True)


@pytest.mark.parametrize("n,fo,k", [(20, 48, 96), (600, 200, 300), (600, 2000, 512)])
def test_product_of_rows_outside_the_segments_and_specials(n, fo, k):
    x, seg, codes, scales, _ = check_product(n, 2, k, fo)
    out = torch.full((n, fo), 7.0, device=DEV)
    part = torch.tensor([3, 10, n - 2], dtype=torch.int32, device=DEV)
    full = torch.tensor([0, 10, n], dtype=torch.int32, device=DEV)
    want = mp.mx_segment_matmul(full, x, codes, scales)
    mp.mx_segment_matmul(part, x, codes, scales, out=out)
    assert torch.equal(out[3:-2], want[3:-2])
    assert bool((out[:3] == 7).all()) and bool((out[-2:] == 7).all())
    # a row with an infinity, and a weight block that is NaN, reach their row and column alone
    y = x.clone()
    y[5, k - 1] = float("inf")
    got = mp.mx_segment_matmul(full, y, codes, scales)
    assert bool(got[5].isnan().all()) and torch.equal(got[:5], want[:5]) and torch.equal(got[6:], want[6:])
    nan = scales.clone()
    nan[1, 4, 0] = 255
    got = mp.mx_segment_matmul(full, x, codes, nan)
    assert bool(got[10:, 4].isnan().all()) and torch.equal(got[:10], want[:10])
    assert torch.equal(got[:, :4], want[:, :4]) and torch.equal(got[:, 5:], want[:, 5:])


def test_no_rows_and_empty_segments():
    code, s = weights(3, 16, 64, 1)
    codes, scales = torch.from_numpy(ref.mx_pack(code)).to(DEV), torch.from_numpy(s.astype(np.uint8)).to(DEV)
    seg = torch.zeros(4, dtype=torch.int32, device=DEV)
    assert mp.mx_segment_matmul(seg, torch.zeros(0, 64, device=DEV), codes, scales).shape == (0, 16)
    out = torch.full((5, 16), 7.0, device=DEV)
    mp.mx_segment_matmul(seg, torch.ones(5, 64, device=DEV), codes, scales, out=out)
    assert bool((out == 7).all())


def test_weights_from_the_projections_layout():
    """segment_matmul's W [T, F, Fo] quantised along F: its values give the same product."""
    g = torch.Generator().manual_seed(2)
    W = torch.randn(2, 64, 40, generator=g).bfloat16().to(DEV)
    x = rows(50, 64, torch.bfloat16, 4)
    Wt = W.transpose(1, 2)
    codes, scales, values = mp.mx_quantize(Wt, want_values=True)
    assert codes.shape == (2, 40, 32) and scales.shape == (2, 40, 2) and values.shape == Wt.shape
    seg = [0, 20, 50]
    _, _, xq = mp.mx_quantize(x, want_values=True)
    a = mp.mx_segment_matmul(torch.tensor(seg, dtype=torch.int32, device=DEV), x, codes, scales)
    b = mp.segment_matmul(seg, xq, values.transpose(1, 2).contiguous())
    size = mp.segment_matmul(seg, xq.abs(), values.abs().transpose(1, 2).contiguous())
    assert bool(((a - b).abs() <= 2.0 ** -18 * size).all())


def test_same_inputs_same_bits_and_side_stream():
    x, seg, codes, scales, out = check_product(600, 3, 256, 300)
    torch.cuda.synchronize()
    s = torch.cuda.Stream()
    again = mp.mx_segment_matmul(seg, x, codes, scales, stream=s)
    torch.cuda.synchronize()
    assert torch.equal(out, again)


def test_refusals():
    x = rows(4, 64, torch.bfloat16, 5)
    seg = torch.tensor([0, 4], dtype=torch.int32, device=DEV)
    codes, scales = mp.mx_quantize(torch.ones(1, 8, 64, device=DEV))
    mp.mx_segment_matmul(seg, x, codes, scales)
    with pytest.raises(ValueError):
        mp.mx_segment_matmul(seg, x[:, :30].contiguous(), codes, scales)
    with pytest.raises(ValueError):
        mp.mx_segment_matmul(seg[:1], x, codes, scales)
    with pytest.raises(ValueError):
        mp.mx_segment_matmul(seg, x, codes, scales[:, :, :1])
    with pytest.raises(ValueError):
        mp.mx_segment_matmul(seg, x, codes.int(), scales)
    with pytest.raises(ValueError):
        mp.mx_segment_matmul(seg, x, codes, scales, out=torch.empty(4, 9, device=DEV))
    with pytest.raises(ValueError):
        mp.mx_segment_matmul(seg, x.half(), codes, scales)
    with pytest.raises(ValueError):
        mp.mx_quantize(x.half())
    with pytest.raises(ValueError):
        mp.mx_dequantize(codes, scales, 65)
    with pytest.raises(mp.MPError):
        mp.mx_quantize(torch.zeros(1, 65537, device=DEV))
