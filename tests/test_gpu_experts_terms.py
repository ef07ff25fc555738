"""The experts of few rows keep fp32 rows and the hidden values whole, whatever the result's type."""
import pytest
import torch

import paper_2507_16991_amd as mp
from test_gpu_experts import BF16, DEV, F32, choices, rows_of, weights
from layer_refs import f64

pytestmark = pytest.mark.gpu

FINE = 1 + 2.0 ** -8 + 2.0 ** -20  # 21 bits: three terms of bf16


def pairs_apart(h):
    """w2 [1, h / 2, h]: the difference of neighbouring hidden values."""
    w = torch.zeros(1, h // 2, h)
    at = torch.arange(h // 2)
    w[0, at, 2 * at], w[0, at, 2 * at + 1] = 1.0, -1.0
    return w.to(BF16).to(DEV)


def as_kind(w, kind):
    return w if kind == "bf16" else mp.mx_quantize(w)


@pytest.mark.parametrize("out", [F32, BF16])
@pytest.mark.parametrize("w", ["bf16", "mx4"])
@pytest.mark.parametrize("x", ["f32", "bf16", "mx8"])
@pytest.mark.parametrize("gated", [False, True])
@pytest.mark.parametrize("n", [1, 20])
def test_hidden_values_are_whole(n, gated, x, w, out):
    """Hidden values 1 + 2^-8 + 2^-20 and 1 + 2^-8, added up from exact products: their difference is 2^-20
    in any order of the sums."""
    h = 48
    rows = torch.zeros(n, 128, device=DEV)
    rows[:, 0], rows[:, 32], rows[:, 64], rows[:, 96] = 1.0, 2.0 ** -8, 2.0 ** -20, 1.0
    w1 = torch.zeros(1, h * (1 + gated), 128, dtype=BF16, device=DEV)
    w1[0, :h, [0, 32]], w1[0, 0:h:2, 64], w1[0, h:, 96] = 1.0, 1.0, 1.0
    if x == "mx8":
        codes = torch.zeros(n, 128, dtype=torch.uint8, device=DEV)
        codes[:, ::32] = 0x38  # 1.0
        rows = codes, torch.tensor([127, 119, 107, 127], dtype=torch.uint8, device=DEV).repeat(n, 1)
    elif x == "bf16":
        rows = rows.to(BF16)
    idx, weight = torch.zeros(n, 1, dtype=torch.int32, device=DEV), torch.ones(n, 1, device=DEV)
    got = mp.expert_mlp(rows, idx, weight, as_kind(w1, w), as_kind(pairs_apart(h), w), act="none", gated=gated,
                        out_dtype=out)
    assert got.dtype == out and (f64(got) == 2.0 ** -20).all()


@pytest.mark.parametrize("out", [F32, BF16])
@pytest.mark.parametrize("w", ["bf16", "mx4"])
@pytest.mark.parametrize("n", [1, 20])
def test_fp32_rows_are_whole(n, w, out):
    """A first product that already takes 1 + 2^-8 from 1 + 2^-8 + 2^-20."""
    x = torch.zeros(n, 64, device=DEV)
    x[:, 3], x[:, 40] = FINE, 1 + 2.0 ** -8
    w1 = torch.zeros(1, 32, 64, dtype=BF16, device=DEV)
    w1[0, :, 3], w1[0, :, 40] = 1.0, -1.0
    w2 = torch.eye(32, device=DEV).to(BF16)[None]
    idx, weight = torch.zeros(n, 1, dtype=torch.int32, device=DEV), torch.ones(n, 1, device=DEV)
    got = mp.expert_mlp(x, idx, weight, as_kind(w1, w), as_kind(w2, w), act="none", gated=False, out_dtype=out)
    assert (f64(got) == 2.0 ** -20).all()


@pytest.mark.parametrize("w", ["bf16", "mx4"])
@pytest.mark.parametrize("x", ["f32", "bf16", "mx8"])
@pytest.mark.parametrize("n", [3, 40])
def test_a_bf16_result_is_the_fp32_one_rounded(n, x, w):
    w1, _ = weights(6, 2 * 200, 300, w, 1)
    w2, _ = weights(6, 130, 200, w, 2)
    rows, _ = rows_of(n, 300, x, 3)
    idx, weight = choices(n, 6, 3, 4)
    whole = mp.expert_mlp(rows, idx, weight, w1, w2, out_dtype=F32)
    assert torch.equal(mp.expert_mlp(rows, idx, weight, w1, w2, out_dtype=BF16), whole.to(BF16))


@pytest.mark.parametrize("out", [F32, BF16])
@pytest.mark.parametrize("w", ["bf16", "mx4"])
@pytest.mark.parametrize("x", ["f32", "bf16", "mx8"])
@pytest.mark.parametrize("at", [0, 64, 130])
@pytest.mark.parametrize("n", [1, 20])
def test_small_products_beside_large_ones(n, at, x, w, out):
    """448 * 6 + 2^-6 / 2 + 448 * -6 of neighbouring places: the sums have at most 20 bits, and the small
    product is left of the large ones."""
    k = 192
    rows = torch.zeros(n, k, device=DEV)
    rows[:, at], rows[:, at + 1], rows[:, at + 2] = 448.0, 2.0 ** -6, 448.0
    if x == "mx8":
        codes = rows.to(torch.float8_e4m3fn).view(torch.uint8)
        rows = codes, torch.full((n, k // 32), 127, dtype=torch.uint8, device=DEV)
    elif x == "bf16":
        rows = rows.to(BF16)
    w1 = torch.zeros(1, 32, k, dtype=BF16, device=DEV)
    w1[0, :, at], w1[0, :, at + 1], w1[0, :, at + 2] = 6.0, 0.5, -6.0
    w2 = torch.eye(32, device=DEV).to(BF16)[None]
    idx, weight = torch.zeros(n, 1, dtype=torch.int32, device=DEV), torch.ones(n, 1, device=DEV)
    got = mp.expert_mlp(rows, idx, weight, as_kind(w1, w), as_kind(w2, w), act="none", gated=False, out_dtype=out)
    assert (f64(got) == 2.0 ** -7).all()
