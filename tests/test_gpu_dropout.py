"""Dropout against the definition in 64 bits: which elements stay is exact; values are one rounded
product (and one fused sum with a residual) in the element type."""
import numpy as np
import pytest
import torch

import layer_refs as ref
import paper_2507_16991_amd as mp

pytestmark = pytest.mark.gpu
DEV = torch.device("cuda:0")
SEED = 0x0123456789ABCDEF
# one rounding of the product (and of the fused sum: relative to the terms) to fp32, and one to bf16
EPS = {torch.float32: 2.0 ** -23, torch.bfloat16: 2.0 ** -8}


def table(n, f, ld, dtype, seed):
    g = torch.Generator().manual_seed(seed)
    t = torch.randn(n, ld, generator=g).to(dtype).to(DEV)
    return t[:, :f]


def check(x, out, p, residual=None, **kw):
    want, keep = ref.dropout(ref.f64(x), p, SEED, residual=None if residual is None else
                             ref.f64(residual), **kw)
    got = ref.f64(out)
    size = np.abs(want) + (0 if residual is None else np.abs(ref.f64(residual)))
    assert np.all(np.abs(got - want) <= EPS[x.dtype] * size)
    if residual is None:
        assert np.array_equal(got != 0, keep & (ref.f64(x) != 0))


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("n,f,pad", [(1, 1, 0), (1, 7, 0), (5, 1, 0), (300, 1, 3), (33, 8, 0),
                                     (17, 13, 0), (17, 13, 6), (129, 64, 0), (40, 100, 28),
                                     (7, 1000, 0), (3, 4099, 1)])
def test_elements(n, f, pad, dtype):
    x, r = table(n, f, f + pad, dtype, 1), table(n, f, f + pad, dtype, 2)
    for p in (0.0, 0.1, 0.5, 1.0):
        check(x, mp.dropout(x, p, SEED, offset=5), p, t=5)
    check(x, mp.dropout(x, 0.3, SEED, residual=r), 0.3, residual=r)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("n,f", [(1, 1), (1000, 1), (257, 8), (100, 13), (31, 100)])
def test_ids_and_rows(n, f, dtype):
    x = table(n, f, f, dtype, 3)
    ids = np.random.default_rng(4).integers(0, 2 ** 31 - 1, n).astype(np.int32)
    d = torch.from_numpy(ids).to(DEV)
    check(x, mp.dropout(x, 0.4, SEED, ids=d), 0.4, ids=ids)
    check(x, mp.dropout(x, 0.4, SEED, ids=d, rows=True), 0.4, ids=ids, rows=True)
    check(x, mp.dropout(x, 0.4, SEED, rows=True), 0.4, rows=True)
    check(x, mp.dropout_backward(x, 0.4, SEED, ids=d), 0.4, ids=ids)


def test_order_of_rows_does_not_matter():
    x = table(500, 24, 24, torch.float32, 5)
    order = torch.randperm(500)
    ids = order.int().to(DEV)
    a = mp.dropout(x, 0.5, SEED)
    b = mp.dropout(x[order.to(DEV)].contiguous(), 0.5, SEED, ids=ids)
    assert torch.equal(a[order.to(DEV)], b)


def test_edge_weights_and_strided_vectors():
    w = table(1001, 1, 1, torch.float32, 6)[:, 0]
    check(w[:, None], mp.dropout(w, 0.25, SEED)[:, None], 0.25)
    s = table(400, 1, 3, torch.float32, 7)[:, 0]
    assert s.stride(0) == 3
    check(s[:, None], mp.dropout(s, 0.25, SEED)[:, None], 0.25)


def test_dropped_elements_are_zero_whatever_they_hold():
    x = torch.full((64, 33), float("nan"), device=DEV)
    x[::2] = float("inf")
    _, keep = ref.dropout(np.ones((64, 33)), 0.5, SEED)
    got = mp.dropout(x, 0.5, SEED).cpu().numpy()
    assert np.all(got[~keep] == 0) and not np.any(np.isfinite(got[keep]))
    assert np.all(mp.dropout(x, 1.0, SEED).cpu().numpy() == 0)


def test_in_place_strided_output_and_untouched_padding():
    x = table(50, 20, 27, torch.bfloat16, 8)
    want = mp.dropout(x, 0.5, SEED)
    out = torch.full((50, 31), 7.0, dtype=torch.bfloat16, device=DEV)
    mp.dropout(x, 0.5, SEED, out=out[:, :20])
    assert torch.equal(out[:, :20], want) and bool((out[:, 20:] == 7).all())
    assert torch.equal(mp.dropout(x, 0.5, SEED, out=x), want) and torch.equal(x, want)


def test_large_counters_and_unaligned_start():
    """Element numbers past 2^32, offsets of 64 bits, and a table that starts at an odd element."""
    base = table(1, 2 * 6000 + 1, 12001, torch.bfloat16, 9)[0, 1:].view(2, 6000)
    ids = np.array([2 ** 31 - 1, 5], np.int32)
    t = 2 ** 40 + 17
    check(base, mp.dropout(base, 0.5, SEED, offset=t, ids=torch.from_numpy(ids).to(DEV)), 0.5,
          ids=ids, t=t)
    check(base, mp.dropout(base, 0.5, SEED, offset=t), 0.5, t=t)


def test_share_of_elements_that_stay():
    n = 1 << 22
    x = torch.ones(n, device=DEV)
    for p in (0.1, 0.5, 0.9):
        kept = float((mp.dropout(x, p, SEED + 1) != 0).double().mean())
        # five standard deviations of a binomial share, and the probability's own step
        assert abs(kept - (1 - p)) < 5 * (p * (1 - p) / n) ** 0.5 + 2.0 ** -17


def test_captured_graph_draws_anew_by_the_step():
    x = table(300, 40, 40, torch.float32, 10)
    step = torch.zeros(1, dtype=torch.int64, device=DEV)
    out = torch.empty_like(x)
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        mp.dropout(x, 0.5, SEED, step=step, out=out)
    torch.cuda.current_stream().wait_stream(s)
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        mp.dropout(x, 0.5, SEED, offset=3, step=step, out=out)
    for k in range(4):
        step.fill_(k)
        g.replay()
        torch.cuda.synchronize()
        assert torch.equal(out, mp.dropout(x, 0.5, SEED, offset=3 + k))
        torch.cuda.synchronize()


def test_side_stream():
    x = table(1000, 64, 64, torch.float32, 11)
    torch.cuda.synchronize()
    s = torch.cuda.Stream()
    out = mp.dropout(x, 0.5, SEED, stream=s)
    s.synchronize()
    check(x, out, 0.5)


def test_same_inputs_same_bits():
    x = table(777, 77, 77, torch.bfloat16, 12)
    assert torch.equal(mp.dropout(x, 0.3, SEED), mp.dropout(x, 0.3, SEED))


def test_refusals():
    x = table(4, 4, 4, torch.float32, 13)
    with pytest.raises(mp.MPError):
        mp.dropout(x, 1.5, SEED)
    with pytest.raises(ValueError):
        mp.dropout(x, 0.5, SEED, ids=torch.zeros(3, dtype=torch.int32, device=DEV))
    with pytest.raises(ValueError):
        mp.dropout(x, 0.5, SEED, ids=torch.zeros(4, dtype=torch.int64, device=DEV))
    with pytest.raises(ValueError):
        mp.dropout(x, 0.5, SEED, residual=x.bfloat16())
    with pytest.raises(ValueError):
        mp.dropout(x.half(), 0.5, SEED)
    with pytest.raises(ValueError):
        mp.dropout(x.t()[:, :2], 0.5, SEED)
