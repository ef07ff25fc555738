"""What lies past the columns of rows in 8 bits."""
import pytest
import torch

import paper_2507_16991_amd as mp

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("f", [1, 5, 24, 33, 200, 1000, 2051, 9001])
def test_codes_past_the_row_are_zero(f, dtype):
    """Also of rows that hold an infinity or NaN, whose every value (or some) is NaN."""
    x = torch.randn(6, f, generator=torch.Generator().manual_seed(f)).to(dtype).to(DEV)
    x[1, f // 2], x[2, 0], x[4, f - 1] = float("nan"), float("inf"), float("-inf")
    codes, scales, values, _ = mp.rms_norm_mx8(x, want_values=True)
    assert not codes[:, f:].any()
    nan = values.isnan()
    assert nan[1].all() and (scales[1] == 255).all()
    for r, c in ((2, 0), (4, f - 1)):
        block = slice(c // 32 * 32, c // 32 * 32 + 32)
        assert nan[r, block].all() and int(nan[r].sum()) == nan[r, block].numel() and scales[r, c // 32] == 255
    assert not nan[[0, 3, 5]].any()


def test_a_row_of_nan_reaches_no_other_through_the_experts():
    x = torch.randn(4, 40, generator=torch.Generator().manual_seed(1)).to(DEV)
    codes, scales, _, _ = mp.rms_norm_mx8(x)
    w1 = torch.ones(1, 8, 40, dtype=torch.bfloat16, device=DEV)
    w2 = torch.ones(1, 8, 8, dtype=torch.bfloat16, device=DEV)
    idx, weight = torch.zeros(4, 1, dtype=torch.int32, device=DEV), torch.ones(4, 1, device=DEV)
    want = mp.expert_mlp((codes, scales), idx, weight, w1, w2, gated=False)
    x[2, 7] = float("nan")
    codes, scales, _, _ = mp.rms_norm_mx8(x)
    got = mp.expert_mlp((codes, scales), idx, weight, w1, w2, gated=False)
    assert torch.equal(got[[0, 1, 3]], want[[0, 1, 3]]) and got[2].isnan().all()
