"""The softmax router against its definition in 64 bits.  Choices and counts are exact; a weight or
probability carries the rounding of its exponent (logit difference, 2^-24 of it), of the exponential
and of a sum of E terms."""
import numpy as np
import pytest
import torch

import layer_refs as ref
import paper_2507_16991_amd as mp

pytestmark = pytest.mark.gpu
DEV = torch.device("cuda:0")


def tolerance(l, E):
    fin = l[np.isfinite(l)]
    span = float(fin.max() - fin.min()) if fin.size else 0.0
    return (8 + 2 * span + E / 2) * 2.0 ** -23


def logits(n, e, dtype, seed, spread=2.0):
    g = torch.Generator().manual_seed(seed)
    return (spread * torch.randn(n, e, generator=g)).to(dtype).to(DEV)


def check(x, k, mask=None, renorm=True, seed=0, backward=True):
    n, e = x.shape
    l = ref.f64(x)
    m = None if mask is None else mask.cpu().numpy()
    idx_r, part = ref.choose(l, k, m)
    l = np.where(part[:, None], l, 0.0)
    w_r, counts_r, rows, loss_r, p, lse = ref.route(l, idx_r, part, renorm)
    idx, weight, counts, loss = mp.route(x, k, mask=mask, renorm=renorm)
    assert np.array_equal(idx.cpu().numpy(), idx_r)
    assert np.array_equal(counts.cpu().numpy(), np.append(counts_r, rows))
    tol = tolerance(l[part], e)
    finite = np.where(np.isfinite(l), np.abs(l), 0.0)
    assert np.all(np.abs(ref.f64(weight) - w_r) <= tol * w_r + 1e-37)
    got = ref.f64(loss)
    assert abs(got[0] - loss_r[0]) <= (tol + 40 * 2.0 ** -23) * loss_r[0]
    # logsumexp: the rounding of the logarithm and of its sum with the maximum
    size = (np.abs(lse) + finite.max(initial=0, axis=1) + 1)[part]
    assert abs(got[1] - loss_r[1]) <= (tol + 40 * 2.0 ** -23) * float((size ** 2).sum()) / max(1, rows)
    if not backward:
        return
    r = np.random.default_rng(seed)
    dw = torch.from_numpy(r.standard_normal((n, k)).astype(np.float32)).to(DEV)
    dl = torch.tensor([0.7 * max(n, 1), -0.3 * max(n, 1)], device=DEV)
    g_r, size = ref.route_backward(l, idx_r, part, ref.f64(dw), ref.f64(dl), renorm)
    g = ref.f64(mp.route_backward(x, idx, weight, counts, dweight=dw, dloss=dl, mask=mask,
                                  renorm=renorm))
    out = 2.0 ** -8 if x.dtype == torch.bfloat16 else 0.0
    lsesize = 1 + finite.max(initial=0)
    bound = 4 * (tol + 8 * 2.0 ** -23) * size * lsesize + out * np.abs(g_r) + 1e-37
    assert np.all(np.abs(g - g_r) <= bound)
    assert np.all(g[~part] == 0)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("n,e,k", [(1, 1, 1), (1, 64, 8), (3, 2, 2), (70, 5, 2), (129, 8, 1),
                                   (65, 13, 13), (1000, 16, 2), (300, 33, 4), (500, 64, 8),
                                   (77, 100, 6), (200, 128, 10), (64, 256, 64), (9, 511, 3),
                                   (50, 513, 8), (21, 1000, 20), (17, 1024, 64)])
def test_sizes(n, e, k, dtype):
    check(logits(n, e, dtype, n + e), k)
    check(logits(n, e, dtype, n + e), k, renorm=False)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("e,k", [(4, 2), (64, 8), (300, 5)])
def test_masks_and_excluded_experts(e, k, dtype):
    x = logits(400, e, dtype, 3)
    mask = torch.rand(400, generator=torch.Generator().manual_seed(5)).to(DEV) < 0.7
    x[~mask] = float("nan")  # whatever was there
    x[torch.rand(400, e, generator=torch.Generator().manual_seed(6)).to(DEV) < 0.2] = -float("inf")
    x[7] = -float("inf")     # nothing to choose
    x[8, :-1] = -float("inf")
    x[9, 1:] = -float("inf")
    mask[7:10] = True
    x[8, -1] = 0.5
    x[9, 0] = -2.0
    check(x, k, mask=mask)
    check(x, k, mask=mask.to(torch.uint8), renorm=False)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_ties_and_signed_zeros(dtype):
    x = torch.randint(-2, 3, (300, 40), generator=torch.Generator().manual_seed(1)).to(dtype).to(DEV)
    x[x == 0] *= torch.where(torch.rand(300, 40, device=DEV)[x == 0] < 0.5, -1.0, 1.0).to(dtype)
    check(x, 8)
    check(torch.zeros(100, 64, dtype=dtype, device=DEV), 8)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_extreme_logits(dtype):
    low = torch.finfo(dtype).min
    x = logits(64, 16, dtype, 8)
    x[:, 3] = low           # the type's lowest value is a logit like any other
    x[1] = low
    x[2] = 80.0
    idx, weight, counts, loss = mp.route(x, 16)
    w = ref.f64(weight)
    assert np.all(np.isfinite(w)) and np.all(np.abs(w.sum(1) - 1) < 1e-5)
    i = idx.cpu().numpy()
    assert i[1].tolist() == list(range(16)) and np.all(w[1] == 1 / 16)
    assert np.all(i[np.arange(64) != 1][:, 15][np.arange(63) != 1] == 3)
    assert np.all(i.sum(1) == 120) and int(counts[16]) == 64


def test_nan_stays_in_its_row_and_in_range():
    x = logits(100, 64, torch.float32, 9)
    x[5, 17] = float("nan")
    idx, weight, counts, loss = mp.route(x, 8)
    assert int(idx.min()) >= 0 and int(idx.max()) < 64
    assert bool(weight[5].isnan().all()) and int(weight.isnan().any(1).sum()) == 1
    assert bool(loss.isnan().all())
    g = mp.route_backward(x, idx, weight, counts, dweight=torch.ones_like(weight))
    assert bool(g[5].isnan().all()) and int(g.isnan().any(1).sum()) == 1


def test_no_rows():
    x = torch.empty(0, 8, device=DEV)
    idx, weight, counts, loss = mp.route(x, 2)
    assert idx.shape == (0, 2) and counts.tolist() == [0] * 9 and loss.tolist() == [0.0, 0.0]
    assert mp.route_backward(x, idx, weight, counts).shape == (0, 8)
    y = logits(10, 8, torch.float32, 1)
    none = torch.zeros(10, dtype=torch.bool, device=DEV)
    idx, weight, counts, loss = mp.route(y, 2, mask=none)
    assert bool((idx == -1).all()) and counts.tolist() == [0] * 9 and loss.tolist() == [0.0, 0.0]
    g = mp.route_backward(y, idx, weight, counts, mask=none, dloss=torch.ones(2, device=DEV))
    assert bool((g == 0).all())


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_strided_logits(dtype):
    x = logits(300, 90, dtype, 11)[:, 5:66]
    assert x.stride(0) == 90
    check(x, 4)


def test_many_rows():
    """Several workgroups, so that their sums are joined."""
    for dtype, n, e, k in ((torch.float32, 30011, 16, 2), (torch.bfloat16, 9001, 64, 8)):
        check(logits(n, e, dtype, 12), k, backward=n < 10000)


@pytest.mark.parametrize("renorm", [True, False])
def test_gradient_against_differences(renorm):
    """The kernel's gradient against central differences of the definition in 64 bits, the choices
    held."""
    x = logits(6, 10, torch.float32, 13, 1.0)
    l = ref.f64(x)
    idx_r, part = ref.choose(l, 3)
    r = np.random.default_rng(2)
    dw, dl = r.standard_normal((6, 3)).astype(np.float32), np.array([3.0, -2.0], np.float32)

    counts_of = ref.route(l, idx_r, part, renorm)[1]

    def f(v):
        w, counts, _, loss, _, _ = ref.route(v, idx_r, part, renorm)
        assert np.array_equal(counts, counts_of)
        return (w * dw).sum() + (loss * dl).sum()

    h = 1e-5
    diff = np.zeros_like(l)
    for i in np.ndindex(l.shape):
        a, b = l.copy(), l.copy()
        a[i] += h
        b[i] -= h
        diff[i] = (f(a) - f(b)) / (2 * h)
    idx, weight, counts, _ = mp.route(x, 3, renorm=renorm)
    g = mp.route_backward(x, idx, weight, counts, dweight=torch.from_numpy(dw).to(DEV),
                          dloss=torch.from_numpy(dl).to(DEV), renorm=renorm)
    # differences: h^2 times a third derivative of order 10, and 1e-16 / h; fp32: 1e-6 of terms of order 10
    assert np.abs(ref.f64(g) - diff).max() < 1e-5


def test_partial_gradients():
    x = logits(50, 12, torch.float32, 14)
    idx, weight, counts, _ = mp.route(x, 2)
    dw = torch.randn(50, 2, device=DEV)
    dl = torch.tensor([2.0, 3.0], device=DEV)
    a = mp.route_backward(x, idx, weight, counts, dweight=dw)
    b = mp.route_backward(x, idx, weight, counts, dloss=dl)
    c = mp.route_backward(x, idx, weight, counts, dweight=dw, dloss=dl)
    assert torch.allclose(a + b, c, rtol=0, atol=1e-5)
    assert bool((mp.route_backward(x, idx, weight, counts) == 0).all())


def test_same_inputs_same_bits_and_side_stream():
    x = logits(20000, 64, torch.float32, 15)
    torch.cuda.synchronize()
    s = torch.cuda.Stream()
    a, b = mp.route(x, 4), mp.route(x, 4, stream=s)
    torch.cuda.synchronize()
    for u, v in zip(a, b):
        assert torch.equal(u, v)


def test_refusals():
    x = logits(4, 8, torch.float32, 16)
    for k in (0, 9, 65):
        with pytest.raises(mp.MPError):
            mp.route(x, k)
    with pytest.raises(mp.MPError):
        mp.route(torch.zeros(2, 1025, device=DEV), 1)
    with pytest.raises(ValueError):
        mp.route(x, 2, mask=torch.ones(3, dtype=torch.bool, device=DEV))
    with pytest.raises(ValueError):
        mp.route(x, 2, mask=torch.ones(4, device=DEV))
    with pytest.raises(ValueError):
        mp.route(x.half(), 2)
    idx, weight, counts, _ = mp.route(x, 2)
    with pytest.raises(ValueError):
        mp.route_backward(x, idx, weight, counts[:-1])
    with pytest.raises(ValueError):
        mp.route_backward(x, idx, weight, counts, dweight=torch.zeros(4, 3, device=DEV))
