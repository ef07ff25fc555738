"""Embedding gradients of wide rows with popular ids, and of many ids in tables past 32 bits."""
import numpy as np
import pytest
import torch

import paper_2507_16991_amd as mp
from test_gpu_embed import BF16, DEV, F32, check_backward, check_forward, make

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("f", [512, 1023, 1500])
@pytest.mark.parametrize("n", [1000, 9000])
def test_a_popular_id_of_wide_rows(n, f, dtype):
    """Most rows are one id's, whose sums come from nearly every workgroup."""
    ids, table, dout = make(n, 5000, f, dtype, torch.int64, spread="even")
    most = torch.rand(n, generator=torch.Generator().manual_seed(n)) < 0.7
    ids[most.to(DEV)] = 2500
    check_forward(ids, table, 1.0, None, mp.embed(ids, table))
    grad = mp.embed_backward(ids, dout, 5000)
    check_backward(ids, dout, 5000, 1.0, None, grad)
    assert torch.equal(grad, mp.embed_backward(ids, dout, 5000))


@pytest.mark.parametrize("n,dtype", [(4000, BF16), (6000, BF16), (6000, F32)])
def test_many_ids_of_tables_past_32_bits(n, dtype):
    """On either side of where few rows are ordered without a sort; most ids are among the last rows."""
    v, f = 2 ** 25 + 77, 70
    g = torch.Generator().manual_seed(n)
    ids = torch.where(torch.rand(n, generator=g) < 0.2, torch.randint(0, v, (n,), generator=g),
                      v - 1 - torch.randint(0, 300, (n,), generator=g))
    ids[:2] = torch.tensor([v - 1, 2 ** 31 // f + 1])
    ids[5:4000:7] = v - 3  # one of several workgroups
    rows = torch.randn(n, f, generator=g).to(dtype).to(DEV)
    present, dense = ids.unique(return_inverse=True)
    ids, present, dense = ids.to(DEV), present.to(DEV), dense.to(DEV)
    grad = mp.embed_backward(ids, rows, v)
    assert grad.numel() > 2 ** 31
    few = mp.embed_backward(dense, rows, len(present))
    check_backward(dense, rows, len(present), 1.0, None, few)
    # (the same order of the rows, and so the same sums)
    assert torch.equal(grad[present], few)
    assert torch.equal(mp.embed(ids, grad), mp.embed(dense, few))
    grad[present] = 0
    assert not grad.any()
