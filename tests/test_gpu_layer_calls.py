"""Calls of the operators around the aggregation at the corners of what the binding accepts: views,
streams, and tables without rows."""
import numpy as np
import pytest
import torch

import layer_refs as ref
import paper_2507_16991_amd as mp

pytestmark = pytest.mark.gpu
DEV = torch.device("cuda:0")


def test_one_row_of_strided_columns_is_refused():
    """As it is for several rows; nothing is read or written beside the view."""
    buf = torch.arange(32, dtype=torch.float32, device=DEV).view(2, 16)
    row, good = buf[:1, ::2], torch.ones(1, 8, device=DEV)
    ptr = torch.tensor([0, 1], dtype=torch.int32, device=DEV)
    codes, scales = mp.mx_quantize(torch.ones(1, 4, 8, device=DEV))
    idx, weight, counts, _ = mp.route(good, 2)
    _, mean, rstd = mp.group_norm(ptr, good, 2)
    calls = [lambda: mp.group_norm(ptr, row, 2), lambda: mp.route(row, 2),
             lambda: mp.group_norm_backward(ptr, row, good, 2, mean, rstd),
             lambda: mp.route_backward(row, idx, weight, counts), lambda: mp.dropout(row, 0.5, 1),
             lambda: mp.dropout(good, 0.5, 1, out=row), lambda: mp.dropout(good, 0.5, 1, residual=row),
             lambda: mp.mx_segment_matmul(ptr, row, codes, scales),
             lambda: mp.spmm(ptr, torch.zeros(1, dtype=torch.int32, device=DEV), row, mp.MP_SUM)]
    for call in calls:
        with pytest.raises(ValueError):
            call()
    assert torch.equal(buf.view(-1).cpu(), torch.arange(32.0))
    # one value has no stride to be wrong about
    assert mp.dropout(buf[1:, 4:10:8], 0.0, 1).tolist() == [[20.0]]


def test_transposed_weights_quantised_on_a_side_stream():
    """What the stream's own earlier work writes is what is quantised, also through a view that has to
    be copied; the copy's memory is not given to other work meanwhile."""
    g = torch.Generator().manual_seed(3)
    W = torch.randn(4, 512, 384, generator=g).bfloat16().to(DEV)
    want = mp.mx_quantize(W.transpose(1, 2).contiguous())
    target = torch.zeros_like(W)
    s = torch.cuda.Stream()
    torch.cuda.synchronize()
    with torch.cuda.stream(s):
        for _ in range(20):  # earlier work that keeps the stream busy
            target.add_(1).sub_(1)
        target.copy_(W)
    got = mp.mx_quantize(target.transpose(1, 2), stream=s)
    for _ in range(4):  # of the copy's size, on the current stream
        torch.full_like(W, 7.0)
    torch.cuda.synchronize()
    for a, b in zip(got, want):
        assert torch.equal(a, b)


def test_one_transposed_weight_is_quantised_as_several_are():
    """Views of a table: transposed, of every second column, repeated, of one row."""
    w = torch.randn(96, 40, generator=torch.Generator().manual_seed(4)).to(DEV)
    for view in (w.t(), w[:, ::2], w[:1, ::2], w[:1].expand(5, 40), w[:, :1].t(), w[:, :1]):
        got = mp.mx_quantize(view, want_values=True)
        want = mp.mx_quantize(view.clone(memory_format=torch.contiguous_format), want_values=True)
        _, scales, values = ref.mx_quantize(ref.f64(view))
        assert np.array_equal(got[1].cpu().numpy(), scales) and np.array_equal(ref.f64(got[2]), values)
        for a, b in zip(got, want):
            assert a.shape == b.shape and torch.equal(a, b)
    empty = mp.mx_quantize(w[:0].t().contiguous().t())
    assert empty[0].shape == (0, 32) and empty[1].shape == (0, 2)


@pytest.mark.parametrize("f,g", [(8, 2), (4096, 1), (4097, 1), (20000, 1), (20000, 4)])
def test_parameter_gradients_of_no_rows_are_zero(f, g):
    """Also of groups too wide for the short path, whose call without rows needs no workspace."""
    x, ptr = torch.empty(0, f, device=DEV), torch.zeros(4, dtype=torch.int32, device=DEV)
    _, mean, rstd = mp.group_norm(ptr, x, g)
    assert bool((mean == 0).all()) and bool((rstd == 0).all())
    dw, db = torch.full((f,), 7.0, device=DEV), torch.full((f,), 7.0, device=DEV)
    nb = mp.mp_group_norm_workspace(0, 3, f, g, mp.MP_F32, 1)
    ws = torch.empty(nb, dtype=torch.uint8, device=DEV) if nb else None
    mp.mp_group_norm_backward(ptr, mp.MP_I32, x, mp.MP_F32, x, 0, 3, f, f, g, None, None, mean, rstd, 0,
                              x, mp.MP_F32, dw, db, ws, nb)
    assert bool((dw == 0).all()) and bool((db == 0).all())
    _, dw, db = mp.group_norm_backward(ptr, x, x, g, mean, rstd)
    assert bool((dw == 0).all()) and bool((db == 0).all())


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("n,s,f,g", [(7, 1, 8, 2), (100, 1, 16, 4), (100, 3, 15, 5), (300, 20, 3, 1),
                                     (20000, 1, 16, 4), (20000, 2, 12, 3), (9000, 2, 6000, 1)])
def test_means_whose_squares_overflow(n, s, f, g, dtype):
    """Equal rows of a power of two past 2^64, whose sums are exact: no variance."""
    top = 2.0 ** 66
    ptr = torch.tensor([n * i // s for i in range(s + 1)], dtype=torch.int32, device=DEV)
    x = torch.full((n, f), top, device=DEV, dtype=dtype)
    x[:, f // 2:] *= -1 if g > 1 and f % (2 * g) == 0 and g % 2 == 0 else 1
    out, mean, rstd = mp.group_norm(ptr, x, g)
    assert bool((out == 0).all()) and bool((mean.abs() == top).all())
    assert torch.allclose(rstd, torch.full_like(rstd, 1e-5 ** -0.5), rtol=1e-6, atol=0)
    dx, dw, db = mp.group_norm_backward(ptr, x, torch.ones_like(x), g, mean, rstd)
    assert all(bool(t.isfinite().all()) for t in (dx, dw, db))


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("n,s,f,g", [(7, 1, 8, 2), (100, 1, 16, 4), (100, 3, 15, 5), (300, 20, 3, 1),
                                     (20000, 1, 16, 4), (20000, 2, 12, 3), (9000, 2, 6000, 1)])
def test_finite_variances_whose_sums_overflow(n, s, f, g, dtype):
    """About means past 2^64, within the rounding of x - mean."""
    top = 2.0 ** 66
    ptr = torch.tensor([n * i // s for i in range(s + 1)], dtype=torch.int32, device=DEV)
    # a spread of 1/64 of the mean: bf16 holds it, and its square is below 2^128 (2^120)
    x = (top * (1 + torch.randn(n, f, generator=torch.Generator().manual_seed(n)) / 64)).to(dtype).to(DEV)
    out, mean, rstd = mp.group_norm(ptr, x, g, out_dtype=torch.float32)
    r = ref.group_norm(ptr.cpu().numpy(), ref.f64(x), g, np.ones(f), np.zeros(f), 1e-5, "none")
    # C u (1 + max|x| rstd) of xhat's size, C = 64 (a run of that many terms): max|x| rstd is below 128
    t = 64 * 2.0 ** -24 * (1 + 128)
    assert np.abs(ref.f64(x)).max() * r["rstd"].max() < 128 or n * f // (s * g) < 64
    if n * f // (s * g) >= 64:
        assert np.all(np.abs(ref.f64(out) - r["out"]) <= t * (1 + np.abs(r["out"])))


@pytest.mark.parametrize("n,s", [(2708, 1), (3000, 200), (60000, 5000), (20000, 3)])
def test_captured_graphs_replay(n, s):
    """Norm, router and 4-bit products, forward and backward, with their workspaces: every replay on new
    inputs gives the bits of the eager calls."""
    f, e, k = 64, 16, 2
    r = np.random.default_rng(n)
    p = np.concatenate([[0], np.sort(r.integers(0, n + 1, s - 1)), [n]]).astype(np.int32)
    ptr = torch.from_numpy(p).to(DEV)
    seg = torch.tensor([0, n // 3, n], dtype=torch.int32, device=DEV)
    short = torch.tensor([0, 7, 20], dtype=torch.int32, device=DEV)
    g = torch.Generator().manual_seed(n)
    x = torch.randn(n, f, generator=g).bfloat16().to(DEV)
    w = torch.randn(f, e, generator=g).to(DEV)
    codes, scales = mp.mx_quantize(torch.randn(2, 48, f, generator=g).to(DEV))

    def step():
        out, mean, rstd = mp.group_norm(ptr, x, 8, act="gelu")
        dx, dw, db = mp.group_norm_backward(ptr, x, out, 8, mean, rstd, act="gelu")
        logits = mp.segment_matmul([0, n], out, w.bfloat16()[None])
        idx, weight, counts, loss = mp.route(logits, k)
        dl = mp.route_backward(logits, idx, weight, counts, dweight=weight, dloss=loss)
        y = mp.mx_segment_matmul(seg, out, codes, scales)
        few = mp.mx_segment_matmul(short, out[:20], codes, scales)
        return [out, mean, rstd, dx, dw, db, idx, weight, counts, loss, dl, y, few]

    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        step()
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        got = step()
    for i in range(4):
        x.copy_(torch.randn(n, f, generator=g).bfloat16())
        want = step()
        graph.replay()
        torch.cuda.synchronize()
        for a, b in zip(got, want):
            assert torch.equal(a, b)
