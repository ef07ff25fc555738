"""Long sums of the experts of few rows against their definition in 64 bits: every number of steps that a
wavefront takes together, and experts of more rows than one product holds."""
import numpy as np
import pytest
import torch

import paper_2507_16991_amd as mp
from test_gpu_experts import BF16, DEV, F32, check, choices, randn, rows_of, weights
from layer_refs import f64

pytestmark = pytest.mark.gpu


def against_the_definition(n, e, k, f, h, fo, x, w, gated=True, act="silu"):
    w1, v1 = weights(e, h * (1 + gated), f, w, 1)
    w2, v2 = weights(e, fo, h, w, 2)
    rows, xv = rows_of(n, f, x, 3)
    if x == "mx8" and w == "mx4":  # the columns that fill a block count as zeros
        pad = -f % 32
        v1, xv = np.pad(v1, ((0, 0), (0, 0), (0, pad))), np.pad(xv, ((0, 0), (0, pad)))
    idx, weight = choices(n, e, k, 4, masked=False)
    out = mp.expert_mlp(rows, idx, weight, w1, w2, act=act, gated=gated, out_dtype=F32)
    check(out, xv, idx, weight, v1, v2, act, gated)
    # (the same sums, rounded once)
    assert torch.equal(mp.expert_mlp(rows, idx, weight, w1, w2, act=act, gated=gated, out_dtype=BF16), out.to(BF16))


# steps of 128 columns for four wavefronts: 1 to 7 whole ones each, with an end of any length or none
@pytest.mark.parametrize("w", ["mx4", "bf16"])
@pytest.mark.parametrize("x", ["f32", "bf16", "mx8"])
@pytest.mark.parametrize("f", [512, 1000, 1536, 2100, 2560, 2561, 3500, 3584])
@pytest.mark.parametrize("n,e", [(16, 1), (49, 1), (64, 3)])
def test_long_rows(n, e, f, x, w):
    against_the_definition(n, e, 1, f, 40, 33, x, w)


# the second product's: steps of an expert's hidden values for the wavefronts of up to 16 workgroups
@pytest.mark.parametrize("w", ["mx4", "bf16"])
@pytest.mark.parametrize("h", [700, 2176, 4099])
@pytest.mark.parametrize("n,e,k", [(1, 2, 2), (16, 1, 1), (49, 1, 1), (64, 3, 2)])
@pytest.mark.parametrize("fo", [20, 600])
def test_long_hidden_rows(n, e, k, h, fo, w):
    against_the_definition(n, e, k, 33, h, fo, "bf16", w, gated=False, act="relu")


@pytest.mark.parametrize("w", ["bf16", "mx4"])
@pytest.mark.parametrize("s", [0, 1, 60, 246, 255])
def test_8_bit_codes_under_extreme_scales(s, w):
    """As with bf16 weights of one: each row holds one code in each of eight blocks."""
    codes = torch.zeros(16, 256, dtype=torch.uint8, device=DEV)
    at = torch.arange(16, device=DEV)
    codes[at, 32 * (at % 8)] = (16 * at + 7).to(torch.uint8)
    scales = torch.full((16, 8), 127, dtype=torch.uint8, device=DEV)
    scales[at, at % 8] = s
    w1 = torch.ones(1, 1, 256, dtype=BF16, device=DEV)
    w2 = torch.ones(1, 1, 1, dtype=BF16, device=DEV) * (2.0 ** 60 if s < 2 else 1.0)
    a, b = (w1, w2) if w == "bf16" else (mp.mx_quantize(w1), mp.mx_quantize(w2))
    idx, weight = torch.zeros(16, 1, dtype=torch.int32, device=DEV), torch.ones(16, 1, device=DEV)
    out = mp.expert_mlp((codes, scales), idx, weight, a, b, act="none", gated=False, out_dtype=F32)
    want = f64(mp.mx8_dequantize(codes, scales, 256)).sum(1) * float(w2)
    # below 2^-126 values are taken in steps of 2^-133, so off by half of one at most; from the scale 3 on
    # they are exact
    tol = 2.0 ** -134 * float(w2) if s < 3 else 0.0
    got = f64(out)[:, 0]
    assert np.array_equal(np.isnan(got), np.isnan(want))
    assert not (np.abs(got - want) > tol).any()


@pytest.mark.parametrize("x", ["f32", "bf16", "mx8"])
@pytest.mark.parametrize("s", [0, 60, 200, 255])
def test_4_bit_codes_under_extreme_scales(s, x):
    """One block of each row of w1 under the scale s, the others under 1; the second product copies h."""
    w1 = torch.zeros(1, 16, 64, dtype=torch.uint8, device=DEV)
    at = torch.arange(16, device=DEV)
    w1[0, at, 16 * (at % 4)] = at.to(torch.uint8)
    scales = torch.full((1, 16, 4), 127, dtype=torch.uint8, device=DEV)
    scales[0, at, at % 4] = s
    eye = mp.mx_quantize(torch.eye(16, device=DEV).to(BF16)[None])
    big = 2.0 ** (100 if s == 0 else 0)
    rows = torch.full((2, 128), big, device=DEV)
    if x == "mx8":
        e = 227 if s == 0 else 127
        rows = torch.full((2, 128), 0x38, dtype=torch.uint8, device=DEV), torch.full((2, 4), e, dtype=torch.uint8, device=DEV)
    elif x == "bf16":
        rows = rows.to(BF16)
    idx, weight = torch.zeros(2, 1, dtype=torch.int32, device=DEV), torch.ones(2, 1, device=DEV)
    out = mp.expert_mlp(rows, idx, weight, (w1, scales), eye, act="none", gated=False, out_dtype=F32)
    h = f64(mp.mx_dequantize(w1, scales, 128))[0].sum(1) * big
    with np.errstate(invalid="ignore"):
        want = (np.eye(16) * h).sum(1)
    # values of 4 bits are k 2^(s - 128), k at most 12: exact in bf16, and their products and sums too
    assert np.isnan(want).any() == (s == 255)
    assert np.array_equal(f64(out), np.stack((want, want)), equal_nan=True)


def test_infinite_and_nan_weights_reach_the_rows_that_chose_them():
    w1, _ = weights(3, 64, 96, "bf16", 1)
    w2, _ = weights(3, 30, 64, "bf16", 2)
    x = randn(3, 6, 96)
    idx, weight = choices(6, 3, 2, 1, masked=False)
    want = mp.expert_mlp(x, idx, weight, w1, w2, gated=False, act="none")
    w1[1, 5, 7], w2[1, 3, 9] = float("nan"), float("inf")
    out = mp.expert_mlp(x, idx, weight, w1, w2, gated=False, act="none")
    hit = (idx == 1).any(1)
    assert 0 < int(hit.sum()) < 6
    assert torch.equal(out[~hit], want[~hit]) and not torch.isfinite(out[hit]).any()
