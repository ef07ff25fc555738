"""The experts of few rows against their definition in 64 bits."""
import numpy as np
import pytest
import torch

import paper_2507_16991_amd as mp
import row_refs as ref
from layer_refs import f64

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
F32, BF16 = torch.float32, torch.bfloat16


def randn(seed, *shape):
    return torch.randn(*shape, generator=torch.Generator().manual_seed(seed)).to(DEV)


def choices(n, e, k, seed, masked=True):
    r = np.random.default_rng([n, e, k, seed])
    idx = np.stack([r.permutation(e)[:k] for _ in range(n)]).astype(np.int32)
    w = r.random((n, k)).astype(np.float32)
    if masked and n > 1:  # a row without any choice, one with a choice less, weights of such places
        idx[r.integers(0, n)] = -1
        idx[r.integers(0, n), k - 1] = -1
    return torch.from_numpy(idx).to(DEV), torch.from_numpy(w).to(DEV)


def weights(e, rows, k, kind, seed):
    """The weights as the call takes them, and their values."""
    w = (randn(seed, e, rows, k) * k ** -0.5).to(BF16)
    if kind == "bf16":
        return w, f64(w)
    codes, scales, values = mp.mx_quantize(w, want_values=True)
    return (codes, scales), f64(values)


def rows_of(n, k, kind, seed):
    if kind == "mx8":
        codes, scales, values, _ = mp.rms_norm_mx8(randn(seed, n, k), want_values=True)
        return (codes, scales), f64(values)
    x = randn(seed, n, k).to(F32 if kind == "f32" else BF16)
    return x, f64(x)


def check(out, x, idx, weight, w1, w2, act, gated, residual=None):
    want, size = ref.expert_mlp(x, idx.cpu().numpy(), f64(weight), w1, w2, act, gated)
    if residual is not None:
        want, size = want + f64(residual), size + np.abs(f64(residual))
    # Sums of K and then k H products: every accumulation of a matrix instruction may round each of its 32
    # additions (2^-23, cut off), over at most K / 32 instructions and the wavefronts' joins; the rest
    # (activation, weights, residual) is 16 half steps.  Under a bf16 result fp32 rows and h are cut to
    # 16 bits (2^-15), and the result is rounded once.
    depth = (x.shape[1] + idx.shape[1] * w2.shape[2] + 64) * 2 + 16
    bf = out.dtype == BF16
    tol = size * (depth * ref.U + (2 * 2.0 ** -15 if bf else 0))
    tol = tol + (np.abs(want) + tol) * (ref.half_step(BF16) if bf else 0)
    assert (np.abs(f64(out) - want) <= tol).all()


@pytest.mark.parametrize("w", ["mx4", "bf16"])
@pytest.mark.parametrize("x", ["f32", "bf16", "mx8"])
@pytest.mark.parametrize("out", [F32, BF16])
@pytest.mark.parametrize("n,e,k,f,h,fo,gated,act", [
    (1, 8, 2, 256, 128, 96, True, "silu"), (1, 1, 1, 1, 1, 1, False, "none"), (3, 5, 2, 33, 17, 31, True, "gelu"),
    (16, 4, 4, 130, 40, 65, False, "relu"), (17, 2, 1, 97, 129, 257, True, "silu"), (64, 3, 2, 160, 96, 33, False, "gelu"),
    (40, 64, 8, 64, 48, 128, True, "relu"), (7, 200, 3, 500, 300, 100, True, "none")])
def test_experts(n, e, k, f, h, fo, gated, act, out, x, w):
    w1, v1 = weights(e, h * (1 + gated), f, w, 1)
    w2, v2 = weights(e, fo, h, w, 2)
    rows, xv = rows_of(n, f, x, 3)
    if x == "mx8" and w == "mx4":  # the columns that fill a block count as zeros
        pad = -f % 32
        v1, xv = np.pad(v1, ((0, 0), (0, 0), (0, pad))), np.pad(xv, ((0, 0), (0, pad)))
    idx, weight = choices(n, e, k, 4)
    res = randn(5, n, fo).to(out)
    got = mp.expert_mlp(rows, idx, weight, w1, w2, act=act, gated=gated, out_dtype=out)
    check(got, xv, idx, weight, v1, v2, act, gated)
    got = mp.expert_mlp(rows, idx, weight, w1, w2, act=act, gated=gated, residual=res, out=torch.empty_like(res))
    check(got, xv, idx, weight, v1, v2, act, gated, res)


@pytest.mark.parametrize("w", ["mx4", "bf16"])
def test_long_sums(w):
    """Many steps of K, of H, and more work than one share of the second product."""
    w1, v1 = weights(3, 2 * 1500, 2100, w, 1)
    w2, v2 = weights(3, 40, 1500, w, 2)
    x = randn(3, 20, 2100).to(BF16)
    idx, weight = choices(20, 3, 2, 1)
    out = mp.expert_mlp(x, idx, weight, w1, w2, out_dtype=F32)
    check(out, f64(x), idx, weight, v1, v2, "silu", True)


def test_wide_and_many_experts():
    w1, v1 = weights(1024, 4, 40, "bf16", 1)
    w2, v2 = weights(1024, 20000 // 512, 4, "bf16", 2)
    x = randn(3, 64, 40)
    idx, weight = choices(64, 1024, 16, 1)
    out = mp.expert_mlp(x, idx, weight, w1, w2, gated=False)
    check(out, f64(x), idx, weight, v1, v2, "silu", False)
    w2, v2 = weights(2, 17000, 16, "mx4", 2)
    w1, v1 = weights(2, 16, 64, "mx4", 1)
    idx, weight = choices(5, 2, 1, 1)
    x = randn(3, 5, 64)
    check(mp.expert_mlp(x, idx, weight, w1, w2, gated=False), f64(x), idx, weight, v1, v2, "silu", False)


def test_no_choice_at_all_and_foreign_numbers():
    w1, v1 = weights(4, 32, 64, "mx4", 1)
    w2, v2 = weights(4, 48, 16, "mx4", 2)
    x = randn(3, 6, 64).to(BF16)
    weight = torch.ones(6, 2, device=DEV)
    none = torch.full((6, 2), -1, dtype=torch.int32, device=DEV)
    res = randn(4, 6, 48).to(BF16)
    assert not mp.expert_mlp(x, none, weight, w1, w2).any()
    assert torch.equal(mp.expert_mlp(x, none, weight, w1, w2, residual=res), res)
    idx = torch.tensor([[0, 4], [-7, 3], [2 ** 31 - 1, -2 ** 31], [1, 2], [5, 0], [3, 3]], dtype=torch.int32,
                       device=DEV)
    check(mp.expert_mlp(x, idx, weight, w1, w2), f64(x), idx, weight, v1, v2, "silu", True)


def test_an_expert_chosen_twice():
    w1, v1 = weights(3, 40, 50, "bf16", 1)
    w2, v2 = weights(3, 60, 20, "bf16", 2)
    x = randn(3, 4, 50)
    idx = torch.tensor([[1, 1, 1], [0, 2, 0], [2, 2, -1], [-1, 1, 1]], dtype=torch.int32, device=DEV)
    weight = torch.rand(4, 3, generator=torch.Generator().manual_seed(1)).to(DEV)
    check(mp.expert_mlp(x, idx, weight, w1, w2), f64(x), idx, weight, v1, v2, "silu", True)


def test_what_is_not_chosen_is_not_read():
    """NaN in other experts' weights, in rows without choices and in weights of no choice."""
    w1, v1 = weights(4, 64, 96, "bf16", 1)
    w2, v2 = weights(4, 30, 32, "bf16", 2)
    x = randn(3, 5, 96)
    idx, weight = choices(5, 3, 2, 1, masked=False)
    idx[2], idx[4, 1] = -1, -1
    want = mp.expert_mlp(x, idx, weight, w1, w2)
    w1[3], w2[3], x[2] = float("nan"), float("nan"), float("nan")
    weight[2], weight[4, 1] = float("nan"), float("inf")
    assert torch.equal(mp.expert_mlp(x, idx, weight, w1, w2), want)


def test_infinities_and_nan_reach_only_their_rows():
    w1, v1 = weights(2, 64, 96, "mx4", 1)
    w2, v2 = weights(2, 30, 64, "mx4", 2)
    x = randn(3, 6, 96)
    idx, weight = choices(6, 2, 2, 1, masked=False)
    want = mp.expert_mlp(x, idx, weight, w1, w2, gated=False, act="none")
    bad = x.clone()
    bad[1, 5], bad[3, 95] = float("inf"), float("nan")
    out = mp.expert_mlp(bad, idx, weight, w1, w2, gated=False, act="none")
    rows = [0, 2, 4, 5]
    assert torch.equal(out[rows], want[rows]) and not torch.isfinite(out[[1, 3]]).any()


@pytest.mark.parametrize("s", [0, 1, 60, 252, 253, 254, 255])
def test_every_code_under_extreme_scales(s):
    """One column of w1 at a time: h is the weight itself, and the second product copies it."""
    codes = torch.zeros(1, 16, 16, dtype=torch.uint8, device=DEV)
    codes[0, :, 0] = torch.arange(16, device=DEV)
    scales = torch.full((1, 16, 1), s, dtype=torch.uint8, device=DEV)
    eye, one = mp.mx_quantize(torch.eye(16, device=DEV).to(BF16)[None])
    x = torch.zeros(1, 32, device=DEV)
    x[0, 0] = 2.0 ** 40 if s < 2 else (2.0 ** -40 if s < 255 else 1.0)
    idx, weight = torch.zeros(1, 1, dtype=torch.int32, device=DEV), torch.ones(1, 1, device=DEV)
    out = mp.expert_mlp(x, idx, weight, (codes, scales), (eye, one), act="none", gated=False)
    # (values past the largest fp32 are infinite, and times the zeros of the second product NaN)
    h = f64(mp.mx_dequantize(codes, scales, 32))[0, :, 0] * float(x[0, 0])
    with np.errstate(invalid="ignore"):
        want = (np.eye(16) * h).sum(1)
    assert np.isfinite(want).all() == (s < 253)
    assert np.array_equal(f64(out)[0], want, equal_nan=True)


@pytest.mark.parametrize("s", [0, 1, 60, 246, 255])
def test_every_8_bit_code_under_extreme_scales(s):
    codes = torch.zeros(16, 256, dtype=torch.uint8, device=DEV)
    at = torch.arange(16, device=DEV)
    codes[at, 32 * (at % 8)] = (16 * at + 7).to(torch.uint8)
    scales = torch.full((16, 8), s, dtype=torch.uint8, device=DEV)
    w1 = torch.ones(1, 1, 256, dtype=BF16, device=DEV)
    w2 = torch.ones(1, 1, 1, dtype=BF16, device=DEV) * (2.0 ** 60 if s < 2 else 1.0)
    idx, weight = torch.zeros(16, 1, dtype=torch.int32, device=DEV), torch.ones(16, 1, device=DEV)
    out = mp.expert_mlp((codes, scales), idx, weight, w1, w2, act="none", gated=False, out_dtype=F32)
    want = f64(mp.mx8_dequantize(codes, scales, 256)).sum(1) * float(w2)
    # Values are taken in bf16, whose steps below 2^-126 are 2^-133: code 7, 7 * 2^-9 2^-127 under the
    # scale 0, lies between two of them and is off by up to half of one, 2^-134.  From the scale 3 on
    # every value is a multiple of 2^-9 2^-124 = 2^-133, and exact.
    tol = 2.0 ** -134 * float(w2) if s < 3 else 0.0
    got = f64(out)[:, 0]
    assert np.array_equal(np.isnan(got), np.isnan(want))
    assert not (np.abs(got - want) > tol).any()


def test_strided_rows_and_in_place_residual():
    w1, _ = weights(4, 64, 70, "bf16", 1)
    w2, _ = weights(4, 70, 32, "bf16", 2)
    x, res = randn(3, 9, 70), randn(4, 9, 70)
    idx, weight = choices(9, 4, 2, 1)
    want = mp.expert_mlp(x, idx, weight, w1, w2, residual=res)
    wide, wide_r = torch.zeros(9, 75, device=DEV), torch.zeros(9, 90, device=DEV)
    wide[:, 3:73], wide_r[:, 5:75] = x, res
    assert torch.equal(mp.expert_mlp(wide[:, 3:73], idx, weight, w1, w2, residual=wide_r[:, 5:75]), want)
    assert torch.equal(mp.expert_mlp(x, idx, weight, w1, w2, residual=res, out=res), want)


def test_no_rows():
    w1, _ = weights(2, 8, 16, "bf16", 1)
    w2, _ = weights(2, 12, 4, "bf16", 2)
    out = mp.expert_mlp(torch.empty(0, 16, device=DEV), torch.empty(0, 2, dtype=torch.int32, device=DEV),
                        torch.empty(0, 2, device=DEV), w1, w2)
    assert out.shape == (0, 12)


def test_same_bits_again_and_on_another_stream():
    w1, _ = weights(16, 2 * 512, 512, "mx4", 1)
    w2, _ = weights(16, 512, 512, "mx4", 2)
    x = randn(3, 33, 512).to(BF16)
    idx, weight = choices(33, 16, 4, 1)
    want = mp.expert_mlp(x, idx, weight, w1, w2)
    for _ in range(5):
        assert torch.equal(mp.expert_mlp(x, idx, weight, w1, w2), want)
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    other = mp.expert_mlp(x, idx, weight, w1, w2, stream=s)
    again = mp.expert_mlp(x, idx, weight, w1, w2)  # (beside it)
    torch.cuda.current_stream().wait_stream(s)
    assert torch.equal(other, want) and torch.equal(again, want)


def test_replayed_from_a_graph():
    w1, _ = weights(8, 2 * 96, 128, "mx4", 1)
    w2, _ = weights(8, 128, 96, "mx4", 2)
    x = randn(3, 12, 128).to(BF16)
    idx, weight = choices(12, 8, 2, 1)

    def step():
        return mp.expert_mlp(x, idx, weight, w1, w2, residual=x)

    step()
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        got = step()
    for seed in range(4):
        x.copy_(randn(seed, 12, 128).to(BF16))
        new = choices(12, 8, 2, seed + 5)
        idx.copy_(new[0])
        weight.copy_(new[1])
        g.replay()
        torch.cuda.synchronize()
        assert torch.equal(got, step())


def test_a_layer_for_few_rows():
    """Embedding, norm in 8 bits, router and experts as they are used together."""
    f, h, e, k, n, v = 256, 128, 8, 2, 11, 500
    table, wr = randn(1, v, f).to(BF16), (randn(2, 1, f, e) / 16).to(BF16)
    (w1, v1), (w2, v2) = weights(e, 2 * h, f, "mx4", 3), weights(e, f, h, "mx4", 4)
    gamma = 1 + 0.1 * randn(5, f)
    ids = torch.randint(0, v, (n,), generator=torch.Generator().manual_seed(6)).to(DEV)
    ids[3] = -1
    x = mp.embed(ids, table, scale=f ** 0.5)
    assert not x[3].any()
    codes, scales, values, _ = mp.rms_norm_mx8(x, gamma, want_values=True)
    logits = mp.segment_matmul([0, n], values, wr)
    idx, weight, counts, _ = mp.route(logits, k, mask=ids >= 0)
    out = mp.expert_mlp((codes, scales), idx, weight, w1, w2, residual=x)
    check(out, f64(values), idx, weight, v1, v2, "silu", True, x)
    assert torch.equal(out[3], x[3])
    # rows of no choice come back as they were, and the router counted the others
    assert int(counts[-1]) == n - 1 and (idx[3] == -1).all()


def test_weights_past_32_bits():
    """The last of experts whose weights take more than 2^32 bytes, against the same expert alone."""
    e, f, h, fo = 5, 16384, 32768, 16000
    w1 = (torch.randint(-8, 9, (e, h, f), device=DEV, dtype=torch.int8)).to(BF16)
    w2 = (torch.randint(-8, 9, (e, fo, h), device=DEV, dtype=torch.int8)).to(BF16)
    assert w1.numel() * 2 > 2 ** 32 and w2.numel() * 2 > 2 ** 32
    x = randn(1, 3, f).to(BF16)
    idx, weight = torch.full((3, 1), e - 1, dtype=torch.int32, device=DEV), torch.ones(3, 1, device=DEV)
    out = mp.expert_mlp(x, idx, weight, w1, w2, act="relu", gated=False)
    alone = mp.expert_mlp(x, idx - (e - 1), weight, w1[e - 1:], w2[e - 1:], act="relu", gated=False)
    assert torch.equal(out, alone) and out.abs().sum() > 0
