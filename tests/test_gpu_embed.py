"""Embedding rows by id and the table's gradient against their definitions in 64 bits."""
import numpy as np
import pytest
import torch

import paper_2507_16991_amd as mp
import row_refs as ref
from layer_refs import f64

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
F32, BF16 = torch.float32, torch.bfloat16


def make(n, v, f, dtype, itype, spread="popular", seed=0, bad=True):
    r = np.random.default_rng([seed, n, v, f])
    u = r.random(n)
    ids = np.minimum((np.exp(u * np.log(v + 1)) - 1 if spread == "popular" else u * v).astype(np.int64),
                     v - 1)
    if spread == "one":
        ids[:] = v // 2
    if bad and n > 2:  # outside the table: padding
        ids[r.integers(0, n)] = -1
        ids[r.integers(0, n)] = v
        ids[r.integers(0, n)] = np.iinfo(np.int32).min if itype == torch.int32 else -2 ** 40
        if itype == torch.int64:
            ids[r.integers(0, n)] = 2 ** 32  # (0 once cut to 32 bits)
    g = torch.Generator().manual_seed(seed)
    table = torch.randn(v, f, generator=g).to(dtype)
    dout = torch.randn(n, f, generator=g).to(dtype)
    return torch.from_numpy(ids).to(itype).to(DEV), table.to(DEV), dout.to(DEV)


def check_forward(ids, table, scale, padding, out):
    want = ref.embed(ids.cpu().numpy().astype(np.int64), f64(table), scale, padding)
    # the product rounded to fp32, then to out's type
    tol = np.abs(want) * (ref.U + ref.half_step(out.dtype) * (1 + ref.U))
    assert (np.abs(f64(out) - want) <= tol).all()


def check_backward(ids, dout, v, scale, padding, grad):
    want, size, count = ref.embed_backward(ids.cpu().numpy().astype(np.int64), f64(dout), v, scale, padding)
    # count additions and the product, each off by half a step of at most the sum of magnitudes
    tol = size * (count[:, None] + 1) * ref.U
    tol = tol + (np.abs(want) + tol) * (ref.half_step(grad.dtype) if grad.dtype == BF16 else 0)
    assert (np.abs(f64(grad) - want) <= tol).all()
    assert not f64(grad)[count == 0].any()


@pytest.mark.parametrize("itype", [torch.int32, torch.int64])
@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("n,v,f", [(1, 1, 1), (1, 7, 128), (3, 5, 3), (65, 300, 7), (64, 64, 8), (1000, 37, 100),
                                   (777, 20011, 33), (5000, 999, 4), (300, 41, 2049), (20000, 3, 1), (17, 9, 65536)])
def test_rows_and_gradient(n, v, f, dtype, itype):
    ids, table, dout = make(n, v, f, dtype, itype)
    check_forward(ids, table, 1.7, None, mp.embed(ids, table, scale=1.7))
    check_backward(ids, dout, v, 1.7, None, mp.embed_backward(ids, dout, v, scale=1.7))


@pytest.mark.parametrize("dtype,out", [(F32, BF16), (BF16, F32)])
def test_other_output_type(dtype, out):
    ids, table, dout = make(500, 90, 50, dtype, torch.int64)
    check_forward(ids, table, 0.3, None, mp.embed(ids, table, scale=0.3, out_dtype=out))
    check_backward(ids, dout, 90, 0.3, None, mp.embed_backward(ids, dout, 90, scale=0.3, out_dtype=out))


# ids of 63, 64 and 65 rows next to each other, and of ranges that begin and end inside of and on the
# borders of the chunks in which long ones are summed
@pytest.mark.parametrize("f", [1, 20, 129, 1500])
@pytest.mark.parametrize("counts", [(64, 64, 64), (65, 63, 65, 64), (1, 127, 65, 190, 1, 64, 66), (200,),
                                    (0, 3, 1000, 0, 0, 700, 5), (64, 65, 64, 129, 128, 127, 0)])
def test_long_and_short_ids(counts, f):
    ids = np.repeat(np.arange(len(counts)), counts)
    ids = np.random.default_rng(5).permutation(ids)
    dout = torch.randn(len(ids), f, generator=torch.Generator().manual_seed(f)).to(DEV)
    t = torch.from_numpy(ids).to(DEV)
    check_backward(t, dout, len(counts), 1.0, None, mp.embed_backward(t, dout, len(counts)))


# either side of where few rows are ordered without a sort, and an id that goes through many workgroups
@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("spread", ["even", "popular", "one"])
@pytest.mark.parametrize("n,v,f", [(2048, 16383, 130), (2049, 16383, 130), (4096, 16384, 40), (4097, 16384, 40), (4095, 99991, 3),
                                   (4096, 20000, 1100)])
def test_few_rows_and_more(n, v, f, spread, dtype):
    ids, _, dout = make(n, v, f, dtype, torch.int64, spread=spread)
    grad = mp.embed_backward(ids, dout, v)
    check_backward(ids, dout, v, 1.0, None, grad)
    assert torch.equal(grad, mp.embed_backward(ids.clamp(-1, v).to(torch.int32), dout, v))


def test_one_id_has_all_rows():
    ids, _, dout = make(70001, 513, 24, BF16, torch.int32, spread="one")
    check_backward(ids, dout, 513, 2.0, None, mp.embed_backward(ids, dout, 513, scale=2.0))


def test_large_batch():
    """Past the sort of small inputs, chunks of more than 64 positions."""
    ids, table, dout = make(1100003, 30011, 5, F32, torch.int64)
    check_forward(ids, table, 1.0, None, mp.embed(ids, table))
    check_backward(ids, dout, 30011, 1.0, None, mp.embed_backward(ids, dout, 30011))


def test_padding_row_holds_anything():
    ids, table, dout = make(400, 30, 40, F32, torch.int64, bad=False)
    table[4] = float("nan")
    dout[ids == 4] = float("inf")
    out = mp.embed(ids, table, padding=4)
    grad = mp.embed_backward(ids, dout, 30, padding=4)
    check_forward(ids, torch.where(table.isnan(), 0, table), 1.0, 4, out)
    check_backward(ids, torch.where(dout.isinf(), 0, dout), 30, 1.0, 4, grad)


def test_everything_is_padding_and_nothing_is_there():
    ids = torch.full((100,), -5, device=DEV, dtype=torch.int64)
    dout = torch.full((100, 12), float("nan"), device=DEV)
    assert not mp.embed(ids, torch.ones(3, 12, device=DEV)).any()
    assert not mp.embed_backward(ids, dout, 3).any()
    none = ids[:0]
    assert mp.embed(none, torch.ones(3, 12, device=DEV)).shape == (0, 12)
    assert not mp.embed_backward(none, dout[:0], 3).any()


def test_strided_rows():
    ids, table, dout = make(300, 50, 24, F32, torch.int32)
    wide_t, wide_d = torch.full((50, 31), 9.0, device=DEV), torch.full((300, 29), 9.0, device=DEV)
    wide_t[:, 3:27], wide_d[:, 1:25] = table, dout
    assert torch.equal(mp.embed(ids, wide_t[:, 3:27]), mp.embed(ids, table))
    assert torch.equal(mp.embed_backward(ids, wide_d[:, 1:25], 50), mp.embed_backward(ids, dout, 50))


def test_same_bits_again_and_on_another_stream():
    ids, table, dout = make(30000, 700, 64, BF16, torch.int64)
    first = mp.embed_backward(ids, dout, 700)
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    other = mp.embed_backward(ids, dout, 700, stream=s)
    rows = mp.embed(ids, table, stream=s)
    torch.cuda.current_stream().wait_stream(s)
    assert torch.equal(first, other) and torch.equal(rows, mp.embed(ids, table))


def test_gradient_is_that_of_the_rows():
    """<dout, embed(table + t d) - embed(table)> = t <dtable, d>: embed is linear in the table."""
    ids, table, dout = make(900, 77, 31, F32, torch.int64)
    grad = mp.embed_backward(ids, dout, 77, scale=3.0)
    d = torch.randn(table.shape, generator=torch.Generator().manual_seed(9)).to(DEV)
    lhs = float((mp.embed(ids, d, scale=3.0).double() * dout.double()).sum())
    size = float((mp.embed(ids, d, scale=3.0).double() * dout.double()).abs().sum())
    # every term is off by a rounding of the forward, and by at most 900 additions in the gradient
    assert abs(lhs - float((grad.double() * d.double()).sum())) <= size * 902 * ref.U


def test_replayed_from_a_graph():
    ids, table, dout = make(20000, 3000, 40, F32, torch.int64)
    out, grad = torch.empty(20000, 40, device=DEV), torch.empty(3000, 40, device=DEV)

    def step():
        mp.embed(ids, table, out=out)
        mp.embed_backward(ids, dout, 3000, out=grad)

    step()
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        step()
    for seed in range(3):
        new = make(20000, 3000, 40, F32, torch.int64, seed=seed + 1)
        for a, b in zip((ids, table, dout), new):
            a.copy_(b)
        g.replay()
        torch.cuda.synchronize()
        assert torch.equal(out, mp.embed(ids, table))
        assert torch.equal(grad, mp.embed_backward(ids, dout, 3000))


def test_tables_past_32_bits():
    v, f = 2 ** 25 + 77, 70
    table = torch.zeros(v, f, dtype=BF16, device=DEV)
    assert table.numel() > 2 ** 31
    rows = torch.randn(500, f, generator=torch.Generator().manual_seed(1)).to(BF16).to(DEV)
    at = torch.randperm(v, generator=torch.Generator().manual_seed(2))[:500]
    at[:3] = torch.tensor([v - 1, 0, 2 ** 31 // f + 1])
    table[at.to(DEV)] = rows
    ids = at.to(DEV)
    assert torch.equal(mp.embed(ids, table), table[ids])
    grad = mp.embed_backward(ids, rows, v)
    assert torch.equal(grad[ids], mp.embed_backward(ids.argsort().argsort(), rows, 500)[ids.argsort().argsort()])
    assert int((grad != 0).any(1).sum()) == len(at.unique())


def test_a_training_step_of_the_entrance():
    """Embedding, residual and norm, and their gradients together, against torch's in 64 bits."""
    n, v, f = 3000, 170, 48
    ids, table, dout = make(n, v, f, F32, torch.int64)
    res = torch.randn(n, f, generator=torch.Generator().manual_seed(3)).to(DEV)
    w = 1 + 0.1 * torch.randn(f, generator=torch.Generator().manual_seed(4)).to(DEV)
    x = mp.embed(ids, table, scale=2.0)
    out, total, rstd = mp.rms_norm(x, w, residual=res)
    dx, dw = mp.rms_norm_backward(total, dout, rstd, w, dtotal=res)
    dtable = mp.embed_backward(ids, dx, v, scale=2.0)

    t64, w64 = table.cpu().double().requires_grad_(), w.cpu().double().requires_grad_()
    i = ids.cpu()
    ok = ((i >= 0) & (i < v))[:, None]
    x64 = torch.where(ok, t64[torch.where(ok[:, 0], i, 0)] * 2.0, 0.0) + res.cpu().double()
    y = x64 / torch.sqrt((x64 ** 2).mean(1, keepdim=True) + float(np.float32(1e-5))) * w64
    ((y * dout.cpu().double()).sum() + (x64 * res.cpu().double()).sum()).backward()
    # dx is off by 237 half steps of its terms (as tested by itself) and, for the two roundings of total
    # (its own and the embedding's), by six times their change; dtable by its additions besides
    _, size, _, sdw = ref.rms_norm_backward(f64(total), f64(dout), f64(w), 1e-5, f64(res))
    _, part, count = ref.embed_backward(i.numpy(), size, v, 2.0)
    tol = part * (237 + 12 + count[:, None] + 1) * ref.U
    assert (np.abs(f64(dtable) - t64.grad.numpy()) <= tol).all()
    assert (np.abs(f64(dw) - w64.grad.numpy()) <= sdw * (n + 50 + 6) * ref.U).all()


@pytest.mark.parametrize("n", [16385, 20480, 20481, 2 ** 20, 2 ** 20 + 1])
@pytest.mark.parametrize("rows", [300, 70001])
def test_order_of_the_sort_on_either_side_of_its_tiles(n, rows):
    """Keys of many and of few equal ones, with and without their numbers carried along."""
    g = torch.Generator().manual_seed(n)
    dst = (torch.rand(n, generator=g) ** 3 * rows).int().clamp(max=rows - 1).to(DEV)
    src = torch.randint(0, 2 ** 20, (n,), generator=g, dtype=torch.int32).to(DEV)
    order = torch.from_numpy(np.argsort(dst.cpu().numpy(), kind="stable")).to(DEV)
    ends = torch.cumsum(torch.bincount(dst, minlength=rows), 0).int()
    for ids in (False, True):
        rowptr, col, perm, _ = mp.coo_to_csr(src, dst, rows, want_perm=ids)
        assert torch.equal(rowptr[1:], ends) and int(rowptr[0]) == 0
        assert torch.equal(col, src[order])
        assert perm is None or torch.equal(perm.long(), order)


@pytest.mark.parametrize("f", [1, 3, 8])
def test_an_id_over_many_short_runs(f):
    """Sums of narrow rows lie in LDS by team; one id begins, fills and ends any number of teams."""
    n, v = 20000, 5000
    for first, length in ((0, n), (3, 8 * 70), (17, 8 * 9 + 5), (2043, 10), (2047, 4098), (5, 2043)):
        ids = torch.arange(n) % 4
        ids[first:first + length] = 4
        ids[first + length:] += 5
        dout = torch.randn(n, f, generator=torch.Generator().manual_seed(length))
        check_backward(ids.sort()[0].to(DEV), dout.to(DEV), v, 1.0, None,
                       mp.embed_backward(ids.sort()[0].to(DEV), dout.to(DEV), v))
